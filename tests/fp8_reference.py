"""Plain forms in 64 bits of the e4m3 quantiser, the block-scaled product and the block norm, for the tests."""
import numpy as np
import torch

# the 127 magnitudes of e4m3 (codes 0 .. 126; 127 is NaN), in order
E4M3 = np.array([(m / 8 * 2.0 ** -6) if e == 0 else (1 + m / 8) * 2.0 ** (e - 7) for e in range(16) for m in range(8)][:127])


def round_e4m3(v):
    """float64 -> the nearest e4m3 magnitude with v's sign, a tie to the even code, beyond 448 clamped, NaN kept."""
    a = np.minimum(np.abs(v), 448.0)
    hi = np.clip(np.searchsorted(E4M3, a), 1, 126)
    lo = hi - 1
    dl, dh = a - E4M3[lo], E4M3[hi] - a
    code = np.where(dl < dh, lo, np.where(dh < dl, hi, np.where(lo % 2 == 0, lo, hi)))
    out = np.copysign(E4M3[code], v)
    return np.where(np.isnan(v), np.nan, out)


def quantize(x, block_rows):
    """x float32 [rows, cols] -> (values of the codes float64 [rows, cols], scales float32, groups first), with the
    definition's fp32 roundings."""
    rows, cols = x.shape
    gr, gc = -(-rows // block_rows), -(-cols // 128)
    f = np.zeros((gr * block_rows, gc * 128), np.float32)
    f[:rows, :cols] = x
    f = f.reshape(gr, block_rows, gc, 128)
    with np.errstate(all="ignore"):
        a = np.abs(f).max(axis=(1, 3))                              # a NaN in the group wins
        s = np.maximum(a / np.float32(448), np.float32(2.0 ** -126))
        i = np.float32(1) / s
        v = (f * i[:, None, :, None]).astype(np.float32)
        q = round_e4m3(v.astype(np.float64))
    return q.reshape(gr * block_rows, gc * 128)[:rows, :cols], np.ascontiguousarray(s.T)


def spread(s, block_rows, rows, cols):
    """scales, groups first -> one for each value."""
    s = torch.as_tensor(s).double()
    return s.repeat_interleave(block_rows, 1)[:, :rows].t().repeat_interleave(128, 1)[:, :cols]


def norm(v, kind, weight, bias, eps):
    """kind: 0 none, 1 rms, 2 layer; float64."""
    if kind == 0:
        return v
    if kind == 2:
        v = v - v.mean(1, keepdim=True)
    v = v / torch.sqrt((v * v).mean(1, keepdim=True) + eps)
    if weight is not None:
        v = v * weight
    return v if bias is None else v + bias


def block_norm(x, y, post, pw, pb, gate, rows_per_gate, skip, branch, pre, qw, qb, eps):
    """float64 tensors -> (r, h)"""
    r = skip * x
    if y is not None:
        u = norm(y, post, pw, pb, eps)
        if gate is not None:
            index = torch.arange(len(x)) // rows_per_gate if rows_per_gate else torch.zeros(len(x), dtype=torch.int64)
            u = u * gate[index]
        r = r + branch * u
    return r, (norm(r, pre, qw, qb, eps) if pre else None)
