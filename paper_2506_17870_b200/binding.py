"""ctypes binding of ``libnq_b200.so``: argument marshalling only.

Each ``nq_*`` function below has the name of the C entry point it calls (``include/nq.h``); it
takes torch CUDA tensors, checks their dtype / device, allocates the outputs through torch and passes
raw device pointers plus the current torch stream to the library.  No step of the computation runs
here, and there is no fallback: if the shared library cannot be loaded the import of a function
raises ``NqLibraryError``.
"""
from __future__ import annotations

import ctypes
from pathlib import Path
from typing import Optional, Sequence

import torch

_PKG = Path(__file__).resolve().parent
_LIB_PATH = _PKG / "libnq_b200.so"
_lib = None

NQ_OK = 0
NQ_F32, NQ_BF16, NQ_E4M3, NQ_I8 = 0, 1, 2, 3
NQ_NORM_NONE, NQ_NORM_RMS, NQ_NORM_LAYER = 0, 1, 2

EXPORTS = (
    "nq_status_str", "nq_low_bits", "nq_packed_row_bytes", "nq_packed_bytes",
    "nq_decompose", "nq_recompose", "nq_drop_low", "nq_unpack", "nq_pack",
    "nq_word64_row_words", "nq_word64_to_sliced", "nq_sliced_to_word64", "nq_rounding_mask",
    "nq_batch_table_bytes", "nq_batch_plan", "nq_recompose_batched", "nq_drop_low_batched",
    "nq_gemm_full", "nq_gemm_part", "nq_conv_workspace_bytes", "nq_conv_implicit_gemm",
    "nq_conv_implicit_gemm_static",
    "nq_gemm_full_q8", "nq_gemm_part_q8", "nq_conv_implicit_gemm_q8", "nq_gemm_nested", "nq_conv_implicit_gemm_nested", "nq_gemm_nested_q8",
    "nq_conv_implicit_gemm_nested_q8",
    "nq_i8_mma_ceiling", "nq_debug_set",
    "nq_conv_implicit_gemm_q8_res", "nq_conv_implicit_gemm_nested_q8_res", "nq_maxpool_nhwc_i8", "nq_avgpool_requant_nhwc_i8",
    "nq_fp8_quantize", "nq_fp8_gemm", "nq_block_norm", "nq_block_norm_backward", "nq_block_norm_backward_workspace_bytes",
    "nq_qk_norm_rotate", "nq_kv_cache_write", "nq_kv_cache_read", "nq_paged_attention", "nq_paged_attention_workspace_bytes",
    "nq_prompt_attention",
    "nq_device_status",
)


class NqLibraryError(RuntimeError):
    pass


class NqError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__(f"{what}: {status_str(status)} (nq_status {status})")


class nq_tensor_desc(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("cols", ctypes.c_int64), ("ld", ctypes.c_int64),
                ("packed_high", ctypes.c_void_p), ("packed_low", ctypes.c_void_p), ("w_int", ctypes.c_void_p)]


class nq_conv_desc(ctypes.Structure):
    _fields_ = [(k, ctypes.c_int32) for k in
                ("B", "Cin", "H", "W", "Cout", "R", "S", "stride", "pad", "x_nchw")]


class nq_block_norm_desc(ctypes.Structure):
    _fields_ = ([(k, ctypes.c_int64) for k in
                 ("rows", "cols", "ldx", "ldy", "ldr", "ldh", "lddx", "lddy", "lddr", "lddh", "rows_per_gate")] +
                [(k, ctypes.c_int32) for k in ("x_dtype", "y_dtype", "h_dtype", "post", "pre")] +
                [(k, ctypes.c_float) for k in ("skip_scale", "branch_scale", "eps", "h_scale")])


class nq_qk_desc(ctypes.Structure):
    _fields_ = ([(k, ctypes.c_int64) for k in ("tokens", "ldx", "ldq", "ldk", "angle_rows")] +
                [(k, ctypes.c_int32) for k in ("x_dtype", "y_dtype", "q_heads", "kv_heads", "head_dim", "rotary_dim", "norm", "neighbours")] +
                [("eps", ctypes.c_float)])


class nq_prompt_desc(ctypes.Structure):
    _fields_ = ([(k, ctypes.c_int64) for k in ("seqs", "rows_q", "rows_k", "ldq", "ldk", "ldv", "ldy")] +
                [(k, ctypes.c_int32) for k in ("q_heads", "kv_heads", "head_dim", "causal", "window")] + [("scale", ctypes.c_float)])


# Argument types of the entry points whose calls pass plain numbers: a call of a few microseconds is not spent on
# wrapping each of them.
_P, _L, _I, _F = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_float
_ARGTYPES = {
    "nq_fp8_quantize": (_P, _L, _I, _L, _L, _I, _P, _L, _P, _L, _P, _L, _P, _L, _P),
    "nq_fp8_gemm": (_P, _L, _P, _L, _P, _L, _P, _L, _I, _P, _L, _L, _L, _P, _L, _I, _I, _P),
    "nq_block_norm": (_P,) * 11 + (_L, _P),
    "nq_block_norm_backward": (_P,) * 17 + (_L, _P),
    "nq_block_norm_backward_workspace_bytes": (_P, _I),
    "nq_qk_norm_rotate": (_P,) * 11,
    "nq_kv_cache_write": (_P, _P, _L, _P, _L, _I, _P, _L, _P),
    "nq_kv_cache_read": (_P, _P, _L, _L, _P, _L, _P, _L, _P, _L, _I, _L, _P),
    "nq_paged_attention": (_P, _P, _L, _L, _P, _L, _L, _P, _L, _I, _F, _P, _L, _P, _L, _P),
    "nq_paged_attention_workspace_bytes": (_P, _L, _L, _L),
    "nq_prompt_attention": (_P,) * 8,
}


def lib() -> ctypes.CDLL:
    """The loaded C library.  Raises NqLibraryError when it has not been built."""
    global _lib
    if _lib is None:
        if not _LIB_PATH.exists():
            raise NqLibraryError(
                f"{_LIB_PATH} is missing: build it with `python -m paper_2506_17870_b200.build` "
                "(needs nvcc); there is no CPU fallback")
        try:
            L = ctypes.CDLL(str(_LIB_PATH))
        except OSError as e:  # pragma: no cover
            raise NqLibraryError(f"cannot load {_LIB_PATH}: {e}") from e
        L.nq_status_str.restype = ctypes.c_char_p
        for name in ("nq_packed_row_bytes", "nq_packed_bytes", "nq_batch_table_bytes", "nq_conv_workspace_bytes",
                     "nq_word64_row_words", "nq_block_norm_backward_workspace_bytes", "nq_paged_attention_workspace_bytes"):
            getattr(L, name).restype = ctypes.c_int64
        for name, types in _ARGTYPES.items():
            getattr(L, name).argtypes = types
        _lib = L
    return _lib


def status_str(status: int) -> str:
    return lib().nq_status_str(int(status)).decode()


def _check(status: int, what: str):
    if status != NQ_OK:
        raise NqError(status, what)


def _ptr(t: Optional[torch.Tensor]):
    return ctypes.c_void_p(0 if t is None else t.data_ptr())


def _i64(v):
    return ctypes.c_int64(int(v))


def _stream():
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def _need(t: torch.Tensor, dtype, name: str, ndim: Optional[int] = None):
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    if ndim is not None and t.dim() != ndim:
        raise ValueError(f"{name} must have {ndim} dimensions")
    if t.dim() >= 1 and t.stride(-1) != 1 and t.numel() > 0:
        raise ValueError(f"{name} must be contiguous in its last dimension")


def _ld(t: torch.Tensor) -> int:
    return t.stride(0) if t.dim() == 2 and t.shape[0] > 1 else max(t.shape[-1], 1)


# --------------------------------------------------------------------------- sizes (host, pure)
def nq_low_bits(n_bits: int, h_bits: int, compensate: bool = True) -> int:
    return int(lib().nq_low_bits(n_bits, h_bits, int(bool(compensate))))


def nq_packed_row_bytes(cols: int, bits: int) -> int:
    return int(lib().nq_packed_row_bytes(_i64(cols), bits))


def nq_packed_bytes(rows: int, cols: int, bits: int) -> int:
    return int(lib().nq_packed_bytes(_i64(rows), _i64(cols), bits))


def _empty_packed(rows: int, cols: int, bits: int, device) -> torch.Tensor:
    """Storage of a packed tensor: nq_packed_bytes(rows, cols, bits) bytes, shaped [rows padded to 128, bytes per row]
    (a container only: the layout stores 128 x 128 blocks, a row's bytes are not contiguous)."""
    return torch.empty((-(-rows // 128) * 128, max(nq_packed_row_bytes(cols, bits), 0)), dtype=torch.uint8, device=device)


# --------------------------------------------------------------------------- codec
def nq_decompose(w_int: torch.Tensor, mask: torch.Tensor, n_bits: int, h_bits: int, compensate: bool = True,
                 out_high: Optional[torch.Tensor] = None, out_low: Optional[torch.Tensor] = None):
    """-> (packed_high, packed_low): uint8 storage of the two sliced tensors."""
    _need(w_int, torch.int8, "w_int", 2)
    _need(mask, torch.uint8, "mask", 2)
    if mask.shape != w_int.shape or _ld(mask) != _ld(w_int):
        raise ValueError("mask must have the shape and row pitch of w_int")
    rows, cols = w_int.shape
    lb = nq_low_bits(n_bits, h_bits, compensate)
    if lb < 0:
        raise NqError(2, "nq_decompose")
    hi = out_high if out_high is not None else _empty_packed(rows, cols, h_bits, w_int.device)
    lo = out_low if out_low is not None else _empty_packed(rows, cols, lb, w_int.device)
    _check(lib().nq_decompose(_ptr(w_int), _ptr(mask), _i64(rows), _i64(cols), _i64(_ld(w_int)), n_bits, h_bits,
                              int(bool(compensate)), _ptr(hi), _ptr(lo), _stream()), "nq_decompose")
    return hi, lo


def nq_recompose(packed_high: torch.Tensor, packed_low: torch.Tensor, rows: int, cols: int, n_bits: int, h_bits: int,
                 compensate: bool = True, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    _need(packed_high, torch.uint8, "packed_high")
    _need(packed_low, torch.uint8, "packed_low")
    if out is None:
        out = torch.empty((rows, cols), dtype=torch.int8, device=packed_high.device)
    _need(out, torch.int8, "out", 2)
    _check(lib().nq_recompose(_ptr(packed_high), _ptr(packed_low), _i64(rows), _i64(cols), n_bits, h_bits,
                              int(bool(compensate)), _ptr(out), _i64(_ld(out)), _stream()), "nq_recompose")
    return out


def nq_drop_low(w_int: torch.Tensor, packed_low: torch.Tensor, n_bits: int, h_bits: int, compensate: bool = True,
                out_high: Optional[torch.Tensor] = None) -> torch.Tensor:
    _need(w_int, torch.int8, "w_int", 2)
    _need(packed_low, torch.uint8, "packed_low")
    rows, cols = w_int.shape
    hi = out_high if out_high is not None else _empty_packed(rows, cols, h_bits, w_int.device)
    _check(lib().nq_drop_low(_ptr(w_int), _i64(_ld(w_int)), _ptr(packed_low), _i64(rows), _i64(cols), n_bits, h_bits,
                             int(bool(compensate)), _ptr(hi), _stream()), "nq_drop_low")
    return hi


def nq_unpack(packed: torch.Tensor, bits: int, rows: int, cols: int, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    _need(packed, torch.uint8, "packed")
    if out is None:
        out = torch.empty((rows, cols), dtype=torch.int8, device=packed.device)
    _check(lib().nq_unpack(_ptr(packed), bits, _i64(rows), _i64(cols), _ptr(out), _i64(_ld(out)), _stream()),
           "nq_unpack")
    return out


def nq_pack(values: torch.Tensor, bits: int) -> torch.Tensor:
    _need(values, torch.int8, "values", 2)
    rows, cols = values.shape
    out = _empty_packed(rows, cols, bits, values.device)
    _check(lib().nq_pack(_ptr(values), _i64(_ld(values)), bits, _i64(rows), _i64(cols), _ptr(out), _stream()),
           "nq_pack")
    return out


NQ_ROUND_DOWN, NQ_ROUND_UP, NQ_ROUND_NEAREST = 0, 1, 2


def nq_rounding_mask(w_int: torch.Tensor, n_bits: int, h_bits: int, mode: int) -> torch.Tensor:
    """Rounding mask (uint8 0 / 1, same shape and pitch as w_int) of one of the baseline roundings."""
    _need(w_int, torch.int8, "w_int", 2)
    rows, cols = w_int.shape
    ld = _ld(w_int)
    buf = torch.empty((rows, ld), dtype=torch.uint8, device=w_int.device)
    _check(lib().nq_rounding_mask(_ptr(w_int), _i64(ld), _i64(rows), _i64(cols), n_bits, h_bits, int(mode), _ptr(buf),
                                  _i64(ld), _stream()), "nq_rounding_mask")
    return buf[:, :cols]


def nq_word64_row_words(cols: int, bits: int) -> int:
    return int(lib().nq_word64_row_words(_i64(cols), bits))


def nq_word64_to_sliced(words: torch.Tensor, bits: int, cols: int) -> torch.Tensor:
    """[rows, nq_word64_row_words(cols, bits)] int64 words (the paper's packed-bit tensor) -> sliced tensor."""
    _need(words, torch.int64, "words", 2)
    rows = words.shape[0]
    if not words.is_contiguous() or words.shape[1] != nq_word64_row_words(cols, bits):
        raise ValueError("words must be a dense [rows, nq_word64_row_words(cols, bits)] tensor")
    out = _empty_packed(rows, cols, bits, words.device)
    _check(lib().nq_word64_to_sliced(_ptr(words), bits, _i64(rows), _i64(cols), _ptr(out), _stream()), "nq_word64_to_sliced")
    return out


def nq_sliced_to_word64(packed: torch.Tensor, bits: int, rows: int, cols: int) -> torch.Tensor:
    """Sliced tensor -> [rows, nq_word64_row_words(cols, bits)] int64 words."""
    _need(packed, torch.uint8, "packed")
    if packed.numel() != nq_packed_bytes(rows, cols, bits):
        raise ValueError("packed has the wrong size for (rows, cols, bits)")
    out = torch.empty((rows, nq_word64_row_words(cols, bits)), dtype=torch.int64, device=packed.device)
    _check(lib().nq_sliced_to_word64(_ptr(packed), bits, _i64(rows), _i64(cols), _ptr(out), _stream()), "nq_sliced_to_word64")
    return out


class BatchPlan:
    """Device table of a model's tensors (nq_batch_plan) plus the work-item count the batched calls need."""

    def __init__(self, table: torch.Tensor, count: int, total_units: int, keep: Sequence[torch.Tensor]):
        self.table, self.count, self.total_units, self._keep = table, count, total_units, list(keep)


def nq_batch_plan(tensors: Sequence[dict]) -> BatchPlan:
    """tensors: dicts with 'w_int' (int8 [rows, cols]), 'packed_high', 'packed_low' (uint8)."""
    count = len(tensors)
    arr = (nq_tensor_desc * max(count, 1))()
    keep = []
    device = tensors[0]["w_int"].device if count else torch.device("cuda")
    for i, t in enumerate(tensors):
        w = t["w_int"]
        _need(w, torch.int8, "w_int", 2)
        _need(t["packed_high"], torch.uint8, "packed_high")
        _need(t["packed_low"], torch.uint8, "packed_low")
        arr[i] = nq_tensor_desc(w.shape[0], w.shape[1], _ld(w), t["packed_high"].data_ptr(),
                                t["packed_low"].data_ptr(), w.data_ptr())
        keep += [w, t["packed_high"], t["packed_low"]]
    nbytes = int(lib().nq_batch_table_bytes(arr, count))
    table = torch.empty(nbytes, dtype=torch.uint8, device=device)
    total = ctypes.c_int64(0)
    _check(lib().nq_batch_plan(arr, count, _ptr(table), _i64(nbytes), ctypes.byref(total), _stream()), "nq_batch_plan")
    return BatchPlan(table, count, total.value, keep)


def nq_recompose_batched(plan: BatchPlan, n_bits: int, h_bits: int, compensate: bool = True):
    _check(lib().nq_recompose_batched(_ptr(plan.table), plan.count, _i64(plan.total_units), n_bits, h_bits,
                                      int(bool(compensate)), _stream()), "nq_recompose_batched")


def nq_drop_low_batched(plan: BatchPlan, n_bits: int, h_bits: int, compensate: bool = True):
    _check(lib().nq_drop_low_batched(_ptr(plan.table), plan.count, _i64(plan.total_units), n_bits, h_bits,
                                     int(bool(compensate)), _stream()), "nq_drop_low_batched")


# --------------------------------------------------------------------------- GEMM
def _y_dtype(dtype) -> int:
    if dtype == torch.float32:
        return NQ_F32
    if dtype == torch.bfloat16:
        return NQ_BF16
    raise ValueError("output dtype must be float32 or bfloat16")


def _gemm_outputs(M, N, device, want_acc, y_dtype, acc_out, y_out):
    acc = acc_out if acc_out is not None else (torch.empty((M, N), dtype=torch.int32, device=device) if want_acc else None)
    y = y_out if y_out is not None else (torch.empty((M, N), dtype=y_dtype, device=device) if y_dtype is not None else None)
    return acc, y


def nq_gemm_full(X: torch.Tensor, W: torch.Tensor, w_scale: torch.Tensor, act_scale: float,
                 bias: Optional[torch.Tensor] = None, want_acc: bool = False, y_dtype=torch.float32,
                 acc_out: Optional[torch.Tensor] = None, y_out: Optional[torch.Tensor] = None):
    """-> (acc int32 [M, N] or None, Y [M, N] or None)."""
    _need(X, torch.int8, "X", 2)
    _need(W, torch.int8, "W", 2)
    _need(w_scale, torch.float32, "w_scale", 1)
    M, K = X.shape
    N = W.shape[0]
    if W.shape[1] != K or w_scale.shape[0] != N:
        raise ValueError("shape mismatch")
    acc, y = _gemm_outputs(M, N, X.device, want_acc, y_dtype, acc_out, y_out)
    _check(lib().nq_gemm_full(_ptr(X), _i64(_ld(X)), _ptr(W), _i64(_ld(W)), _ptr(w_scale), ctypes.c_float(act_scale),
                              _ptr(bias), _i64(M), _i64(N), _i64(K), _ptr(acc), _i64(_ld(acc) if acc is not None else 0),
                              _ptr(y), _i64(_ld(y) if y is not None else 0),
                              _y_dtype(y.dtype) if y is not None else NQ_F32, _stream()), "nq_gemm_full")
    return acc, y


def nq_gemm_part(X: torch.Tensor, packed_high: torch.Tensor, N: int, n_bits: int, h_bits: int, w_scale: torch.Tensor,
                 act_scale: float, bias: Optional[torch.Tensor] = None, want_acc: bool = False,
                 y_dtype=torch.float32, acc_out: Optional[torch.Tensor] = None, y_out: Optional[torch.Tensor] = None):
    _need(X, torch.int8, "X", 2)
    _need(packed_high, torch.uint8, "packed_high")
    _need(w_scale, torch.float32, "w_scale", 1)
    M, K = X.shape
    acc, y = _gemm_outputs(M, N, X.device, want_acc, y_dtype, acc_out, y_out)
    _check(lib().nq_gemm_part(_ptr(X), _i64(_ld(X)), _ptr(packed_high), n_bits, h_bits, _ptr(w_scale),
                              ctypes.c_float(act_scale), _ptr(bias), _i64(M), _i64(N), _i64(K), _ptr(acc),
                              _i64(_ld(acc) if acc is not None else 0), _ptr(y), _i64(_ld(y) if y is not None else 0),
                              _y_dtype(y.dtype) if y is not None else NQ_F32, _stream()), "nq_gemm_part")
    return acc, y


def nq_gemm_nested(X: torch.Tensor, packed_high: torch.Tensor, packed_low: torch.Tensor, N: int, n_bits: int,
                   h_bits: int, w_scale: torch.Tensor, act_scale: float, bias: Optional[torch.Tensor] = None,
                   want_acc: bool = False, y_dtype=torch.float32, acc_out: Optional[torch.Tensor] = None,
                   y_out: Optional[torch.Tensor] = None):
    """Full-bit layer computed from the packed higher-bit and compensated lower-bit tensors (no INT8 copy)."""
    _need(X, torch.int8, "X", 2)
    _need(packed_high, torch.uint8, "packed_high")
    _need(packed_low, torch.uint8, "packed_low")
    _need(w_scale, torch.float32, "w_scale", 1)
    M, K = X.shape
    acc, y = _gemm_outputs(M, N, X.device, want_acc, y_dtype, acc_out, y_out)
    _check(lib().nq_gemm_nested(_ptr(X), _i64(_ld(X)), _ptr(packed_high), _ptr(packed_low), n_bits, h_bits,
                                _ptr(w_scale), ctypes.c_float(act_scale), _ptr(bias), _i64(M), _i64(N), _i64(K),
                                _ptr(acc), _i64(_ld(acc) if acc is not None else 0), _ptr(y),
                                _i64(_ld(y) if y is not None else 0),
                                _y_dtype(y.dtype) if y is not None else NQ_F32, _stream()), "nq_gemm_nested")
    return acc, y


# --------------------------------------------------------------------------- convolution
def nq_gemm_full_q8(X: torch.Tensor, W: torch.Tensor, w_scale: torch.Tensor, act_scale: float, out_scale: float,
                    relu: bool = True, bias: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Full-bit layer whose output is the next layer's INT8 activations."""
    _need(X, torch.int8, "X", 2); _need(W, torch.int8, "W", 2); _need(w_scale, torch.float32, "w_scale", 1)
    M, K = X.shape
    N = W.shape[0]
    y = torch.empty((M, N), dtype=torch.int8, device=X.device)
    _check(lib().nq_gemm_full_q8(_ptr(X), _i64(_ld(X)), _ptr(W), _i64(_ld(W)), _ptr(w_scale), ctypes.c_float(act_scale),
                                 _ptr(bias), ctypes.c_float(out_scale), int(bool(relu)), _i64(M), _i64(N), _i64(K),
                                 _ptr(y), _i64(N), _stream()), "nq_gemm_full_q8")
    return y


def nq_gemm_part_q8(X: torch.Tensor, packed_high: torch.Tensor, N: int, n_bits: int, h_bits: int, w_scale: torch.Tensor,
                    act_scale: float, out_scale: float, relu: bool = True, bias: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Part-bit layer whose output is the next layer's INT8 activations."""
    _need(X, torch.int8, "X", 2); _need(packed_high, torch.uint8, "packed_high"); _need(w_scale, torch.float32, "w_scale", 1)
    M, K = X.shape
    y = torch.empty((M, N), dtype=torch.int8, device=X.device)
    _check(lib().nq_gemm_part_q8(_ptr(X), _i64(_ld(X)), _ptr(packed_high), n_bits, h_bits, _ptr(w_scale),
                                 ctypes.c_float(act_scale), _ptr(bias), ctypes.c_float(out_scale), int(bool(relu)),
                                 _i64(M), _i64(N), _i64(K), _ptr(y), _i64(N), _stream()), "nq_gemm_part_q8")
    return y


def nq_conv_implicit_gemm_q8(X: torch.Tensor, Wt: torch.Tensor, desc: nq_conv_desc, w_scale: torch.Tensor, act_scale: float,
                             out_scale: float, relu: bool = True, part_bit: bool = False, n_bits: int = 8, h_bits: int = 6,
                             bias: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                             y_out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Convolution whose NHWC output is the next layer's INT8 activations."""
    Ho = (desc.H + 2 * desc.pad - desc.R) // desc.stride + 1
    Wo = (desc.W + 2 * desc.pad - desc.S) // desc.stride + 1
    need = nq_conv_workspace_bytes(desc)
    if workspace is None:
        workspace = torch.empty(max(need, 0) + 2048, dtype=torch.uint8, device=X.device)
    off = (-workspace.data_ptr()) % 1024
    y = y_out if y_out is not None else torch.empty((desc.B, Ho, Wo, desc.Cout), dtype=torch.int8, device=X.device)
    ldw = _ld(Wt) if not part_bit else 0
    _check(lib().nq_conv_implicit_gemm_q8(_ptr(X), _ptr(Wt), _i64(ldw), int(bool(part_bit)), n_bits, h_bits,
                                          ctypes.byref(desc), _ptr(w_scale), ctypes.c_float(act_scale), _ptr(bias),
                                          ctypes.c_float(out_scale), int(bool(relu)), _ptr(y),
                                          ctypes.c_void_p(workspace.data_ptr() + off), _i64(workspace.numel() - off),
                                          _stream()), "nq_conv_implicit_gemm_q8")
    return y


def nq_gemm_nested_q8(X: torch.Tensor, packed_high: torch.Tensor, packed_low: torch.Tensor, N: int, n_bits: int,
                      h_bits: int, w_scale: torch.Tensor, act_scale: float, out_scale: float, relu: bool = True,
                      bias: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Nested full-bit layer whose output is the next layer's INT8 activations."""
    _need(X, torch.int8, "X", 2); _need(packed_high, torch.uint8, "packed_high"); _need(packed_low, torch.uint8, "packed_low")
    _need(w_scale, torch.float32, "w_scale", 1)
    M, K = X.shape
    y = torch.empty((M, N), dtype=torch.int8, device=X.device)
    _check(lib().nq_gemm_nested_q8(_ptr(X), _i64(_ld(X)), _ptr(packed_high), _ptr(packed_low), n_bits, h_bits,
                                   _ptr(w_scale), ctypes.c_float(act_scale), _ptr(bias), ctypes.c_float(out_scale),
                                   int(bool(relu)), _i64(M), _i64(N), _i64(K), _ptr(y), _i64(N), _stream()),
           "nq_gemm_nested_q8")
    return y


def nq_conv_implicit_gemm_nested_q8(X: torch.Tensor, packed_high: torch.Tensor, packed_low: torch.Tensor,
                                    desc: nq_conv_desc, w_scale: torch.Tensor, act_scale: float, out_scale: float,
                                    relu: bool = True, n_bits: int = 8, h_bits: int = 6,
                                    bias: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                                    y_out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Nested full-bit convolution whose NHWC output is the next layer's INT8 activations."""
    Ho = (desc.H + 2 * desc.pad - desc.R) // desc.stride + 1
    Wo = (desc.W + 2 * desc.pad - desc.S) // desc.stride + 1
    need = nq_conv_workspace_bytes(desc)
    if workspace is None:
        workspace = torch.empty(max(need, 0) + 2048, dtype=torch.uint8, device=X.device)
    off = (-workspace.data_ptr()) % 1024
    y = y_out if y_out is not None else torch.empty((desc.B, Ho, Wo, desc.Cout), dtype=torch.int8, device=X.device)
    _check(lib().nq_conv_implicit_gemm_nested_q8(_ptr(X), _ptr(packed_high), _ptr(packed_low), n_bits, h_bits,
                                                 ctypes.byref(desc), _ptr(w_scale), ctypes.c_float(act_scale), _ptr(bias),
                                                 ctypes.c_float(out_scale), int(bool(relu)), _ptr(y),
                                                 ctypes.c_void_p(workspace.data_ptr() + off), _i64(workspace.numel() - off),
                                                 _stream()), "nq_conv_implicit_gemm_nested_q8")
    return y


def nq_conv_implicit_gemm_q8_res(X: torch.Tensor, Wt: torch.Tensor, desc: nq_conv_desc, w_scale: torch.Tensor, act_scale: float,
                                 residual: torch.Tensor, residual_scale: float, out_scale: float, relu: bool = True,
                                 part_bit: bool = False, n_bits: int = 8, h_bits: int = 6,
                                 bias: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                                 y_out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Requantising convolution with a residual connection: `residual` (int8, the output's NHWC shape, scale
    residual_scale) is added, dequantised, before the activation."""
    Ho = (desc.H + 2 * desc.pad - desc.R) // desc.stride + 1
    Wo = (desc.W + 2 * desc.pad - desc.S) // desc.stride + 1
    _need(residual, torch.int8, "residual")
    if tuple(residual.shape) != (desc.B, Ho, Wo, desc.Cout) or not residual.is_contiguous():
        raise ValueError("residual must be a dense NHWC tensor of the output's shape")
    need = nq_conv_workspace_bytes(desc)
    if workspace is None:
        workspace = torch.empty(max(need, 0) + 2048, dtype=torch.uint8, device=X.device)
    off = (-workspace.data_ptr()) % 1024
    y = y_out if y_out is not None else torch.empty((desc.B, Ho, Wo, desc.Cout), dtype=torch.int8, device=X.device)
    ldw = _ld(Wt) if not part_bit else 0
    _check(lib().nq_conv_implicit_gemm_q8_res(_ptr(X), _ptr(Wt), _i64(ldw), int(bool(part_bit)), n_bits, h_bits,
                                              ctypes.byref(desc), _ptr(w_scale), ctypes.c_float(act_scale), _ptr(bias),
                                              _ptr(residual), ctypes.c_float(residual_scale), ctypes.c_float(out_scale),
                                              int(bool(relu)), _ptr(y), ctypes.c_void_p(workspace.data_ptr() + off),
                                              _i64(workspace.numel() - off), _stream()), "nq_conv_implicit_gemm_q8_res")
    return y


def nq_conv_implicit_gemm_nested_q8_res(X: torch.Tensor, packed_high: torch.Tensor, packed_low: torch.Tensor,
                                        desc: nq_conv_desc, w_scale: torch.Tensor, act_scale: float,
                                        residual: torch.Tensor, residual_scale: float, out_scale: float,
                                        relu: bool = True, n_bits: int = 8, h_bits: int = 6,
                                        bias: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                                        y_out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The same in nested full-bit mode (weights rebuilt from the two packed parts inside the kernel)."""
    Ho = (desc.H + 2 * desc.pad - desc.R) // desc.stride + 1
    Wo = (desc.W + 2 * desc.pad - desc.S) // desc.stride + 1
    _need(residual, torch.int8, "residual")
    if tuple(residual.shape) != (desc.B, Ho, Wo, desc.Cout) or not residual.is_contiguous():
        raise ValueError("residual must be a dense NHWC tensor of the output's shape")
    need = nq_conv_workspace_bytes(desc)
    if workspace is None:
        workspace = torch.empty(max(need, 0) + 2048, dtype=torch.uint8, device=X.device)
    off = (-workspace.data_ptr()) % 1024
    y = y_out if y_out is not None else torch.empty((desc.B, Ho, Wo, desc.Cout), dtype=torch.int8, device=X.device)
    _check(lib().nq_conv_implicit_gemm_nested_q8_res(_ptr(X), _ptr(packed_high), _ptr(packed_low), n_bits, h_bits,
                                                     ctypes.byref(desc), _ptr(w_scale), ctypes.c_float(act_scale), _ptr(bias),
                                                     _ptr(residual), ctypes.c_float(residual_scale), ctypes.c_float(out_scale),
                                                     int(bool(relu)), _ptr(y), ctypes.c_void_p(workspace.data_ptr() + off),
                                                     _i64(workspace.numel() - off), _stream()),
           "nq_conv_implicit_gemm_nested_q8_res")
    return y


def nq_conv_workspace_bytes(desc: nq_conv_desc) -> int:
    return int(lib().nq_conv_workspace_bytes(ctypes.byref(desc)))


def nq_conv_implicit_gemm(X: torch.Tensor, Wt: torch.Tensor, desc: nq_conv_desc, w_scale: torch.Tensor,
                          act_scale: float, part_bit: bool = False, n_bits: int = 8, h_bits: int = 6,
                          bias: Optional[torch.Tensor] = None, want_acc: bool = False, y_dtype=torch.float32,
                          workspace: Optional[torch.Tensor] = None, acc_out: Optional[torch.Tensor] = None,
                          y_out: Optional[torch.Tensor] = None):
    """X int8 NHWC (or NCHW when desc.x_nchw); Wt int8 [Cout, ldw] (full-bit) or sliced uint8 (part-bit).
    -> (acc int32 [B, Ho, Wo, Cout] or None, Y [B, Ho, Wo, Cout] or None, workspace)."""
    _need(X, torch.int8, "X")
    _need(w_scale, torch.float32, "w_scale", 1)
    if part_bit:
        _need(Wt, torch.uint8, "Wt")
        ldw = 0
    else:
        _need(Wt, torch.int8, "Wt", 2)
        ldw = _ld(Wt)
    Ho = (desc.H + 2 * desc.pad - desc.R) // desc.stride + 1
    Wo = (desc.W + 2 * desc.pad - desc.S) // desc.stride + 1
    need = nq_conv_workspace_bytes(desc)
    if need < 0:
        raise NqError(1, "nq_conv_workspace_bytes")
    if workspace is None:
        workspace = torch.empty(max(need, 1024) + 1024, dtype=torch.uint8, device=X.device)
    off = (-workspace.data_ptr()) % 1024
    ws = workspace[off:]
    shape = (desc.B, Ho, Wo, desc.Cout)
    acc = acc_out if acc_out is not None else (torch.empty(shape, dtype=torch.int32, device=X.device) if want_acc else None)
    y = y_out if y_out is not None else (torch.empty(shape, dtype=y_dtype, device=X.device) if y_dtype is not None else None)
    _check(lib().nq_conv_implicit_gemm(_ptr(X), _ptr(Wt), _i64(ldw), int(bool(part_bit)), n_bits, h_bits,
                                       ctypes.byref(desc), _ptr(w_scale), ctypes.c_float(act_scale), _ptr(bias),
                                       _ptr(acc), _ptr(y), _y_dtype(y.dtype) if y is not None else NQ_F32,
                                       _ptr(ws), _i64(ws.numel()), _stream()), "nq_conv_implicit_gemm")
    return acc, y, workspace


def nq_conv_implicit_gemm_nested(X: torch.Tensor, packed_high: torch.Tensor, packed_low: torch.Tensor, desc: nq_conv_desc,
                                 w_scale: torch.Tensor, act_scale: float, n_bits: int = 8, h_bits: int = 6,
                                 bias: Optional[torch.Tensor] = None, want_acc: bool = False, y_dtype=torch.float32,
                                 workspace: Optional[torch.Tensor] = None, y_out: Optional[torch.Tensor] = None):
    """The full-bit convolution computed from the packed higher-bit and compensated lower-bit tensors.
    -> (acc int32 [B, Ho, Wo, Cout] or None, Y [B, Ho, Wo, Cout] or None, workspace)."""
    _need(X, torch.int8, "X")
    _need(packed_high, torch.uint8, "packed_high")
    _need(packed_low, torch.uint8, "packed_low")
    _need(w_scale, torch.float32, "w_scale", 1)
    Ho = (desc.H + 2 * desc.pad - desc.R) // desc.stride + 1
    Wo = (desc.W + 2 * desc.pad - desc.S) // desc.stride + 1
    need = nq_conv_workspace_bytes(desc)
    if need < 0:
        raise NqError(1, "nq_conv_workspace_bytes")
    if workspace is None:
        workspace = torch.empty(max(need, 1024) + 1024, dtype=torch.uint8, device=X.device)
    off = (-workspace.data_ptr()) % 1024
    ws = workspace[off:]
    shape = (desc.B, Ho, Wo, desc.Cout)
    acc = torch.empty(shape, dtype=torch.int32, device=X.device) if want_acc else None
    y = y_out if y_out is not None else (torch.empty(shape, dtype=y_dtype, device=X.device) if y_dtype is not None else None)
    _check(lib().nq_conv_implicit_gemm_nested(_ptr(X), _ptr(packed_high), _ptr(packed_low), n_bits, h_bits,
                                              ctypes.byref(desc), _ptr(w_scale), ctypes.c_float(act_scale), _ptr(bias),
                                              _ptr(acc), _ptr(y), _y_dtype(y.dtype) if y is not None else NQ_F32,
                                              _ptr(ws), _i64(ws.numel()), _stream()), "nq_conv_implicit_gemm_nested")
    return acc, y, workspace


NQ_CONV_STATIC_SCRATCH_BYTES = 16 * 1024 * 1024


def nq_conv_implicit_gemm_static(X: torch.Tensor, Wt: torch.Tensor, desc: nq_conv_desc, w_scale: torch.Tensor,
                                 act_scale: float, acc_out: Optional[torch.Tensor], y_out: Optional[torch.Tensor],
                                 part_bit: bool = False, n_bits: int = 8, h_bits: int = 6,
                                 bias: Optional[torch.Tensor] = None):
    """The convolution for callers that cannot allocate: no workspace argument, and this wrapper allocates
    nothing either -- the caller passes the output tensors (acc_out int32 and / or y_out fp32 / bf16, NHWC).
    Layers that need more than NQ_CONV_STATIC_SCRATCH_BYTES of staging raise NqError(NQ_ERR_WORKSPACE)."""
    _need(X, torch.int8, "X")
    _need(w_scale, torch.float32, "w_scale", 1)
    if acc_out is None and y_out is None:
        raise ValueError("pass acc_out and / or y_out")
    if part_bit:
        _need(Wt, torch.uint8, "Wt")
        ldw = 0
    else:
        _need(Wt, torch.int8, "Wt", 2)
        ldw = _ld(Wt)
    _check(lib().nq_conv_implicit_gemm_static(_ptr(X), _ptr(Wt), _i64(ldw), int(bool(part_bit)), n_bits, h_bits,
                                              ctypes.byref(desc), _ptr(w_scale), ctypes.c_float(act_scale), _ptr(bias),
                                              _ptr(acc_out), _ptr(y_out),
                                              _y_dtype(y_out.dtype) if y_out is not None else NQ_F32, _stream()),
           "nq_conv_implicit_gemm_static")
    return acc_out, y_out


NQ_DEBUG_PLAIN_STORES, NQ_DEBUG_PACKED_RING = 0, 1


def nq_debug_set(which: int, enabled: bool) -> None:
    """Test aid: force ordinary stores / the packed-tile ring (see nq.h)."""
    _check(lib().nq_debug_set(int(which), int(bool(enabled))), "nq_debug_set")


def nq_maxpool_nhwc_i8(X: torch.Tensor, ksize: int, stride: int, pad: int, y_out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """INT8 NHWC [B, H, W, C] -> [B, Ho, Wo, C], integer maximum over the taps inside the image."""
    _need(X, torch.int8, "X", 4)
    B, H, W, C = X.shape
    Ho, Wo = (H + 2 * pad - ksize) // stride + 1, (W + 2 * pad - ksize) // stride + 1
    y = y_out if y_out is not None else torch.empty((B, Ho, Wo, C), dtype=torch.int8, device=X.device)
    _check(lib().nq_maxpool_nhwc_i8(_ptr(X), B, H, W, C, ksize, stride, pad, _ptr(y), _stream()), "nq_maxpool_nhwc_i8")
    return y


def nq_avgpool_requant_nhwc_i8(X: torch.Tensor, in_scale: float, out_scale: float,
                               y_out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """INT8 NHWC [B, H, W, C] -> INT8 [B, C]: global average, requantised."""
    _need(X, torch.int8, "X", 4)
    B, H, W, C = X.shape
    y = y_out if y_out is not None else torch.empty((B, C), dtype=torch.int8, device=X.device)
    _check(lib().nq_avgpool_requant_nhwc_i8(_ptr(X), B, H, W, C, ctypes.c_float(in_scale), ctypes.c_float(out_scale),
                                            _ptr(y), _stream()), "nq_avgpool_requant_nhwc_i8")
    return y


# --------------------------------------------------------------------------- e4m3 with a scale for each block of 128
_FLOATS = {torch.float32: NQ_F32, torch.bfloat16: NQ_BF16}
_H_TYPES = {**_FLOATS, torch.float8_e4m3fn: NQ_E4M3, torch.int8: NQ_I8}


def _raw_stream(t: torch.Tensor) -> int:
    """The current stream of the tensor's device, which has to be the current device."""
    index = t.get_device()
    if index != torch._C._cuda_getDevice():
        raise ValueError(f"the tensors are on cuda:{index}, the current device is cuda:{torch._C._cuda_getDevice()}")
    return torch._C._cuda_getCurrentRawStream(index)


def _new(rows: int, cols: int, dtype, device, pitch: Optional[int] = None) -> torch.Tensor:
    # (empty_strided is the cheapest of torch's allocating calls: 1.4 us against 2.3 for torch.empty with a shape)
    return torch.empty_strided((rows, cols), (cols if pitch is None else pitch, 1), dtype=dtype, device=device)


def _on(t: torch.Tensor, name: str, index: int) -> None:
    """Refuses a tensor that is not on the GPU of this index, the first operand's."""
    here = t.get_device()
    if here < 0:
        raise ValueError(f"{name} must be a CUDA tensor")
    if here != index:
        raise ValueError(f"{name} is on cuda:{here}, the first operand on {'the host' if index < 0 else f'cuda:{index}'}")


def _matrix(t: torch.Tensor, name: str, index: int, dtype=None, shape=None) -> int:
    """Checks a [rows, cols] tensor on the GPU of this index, with neighbouring columns; -> its row pitch."""
    if t.dim() != 2 or (shape is not None and t.shape != shape):
        raise ValueError(f"{name} must be a {'[rows, cols]' if shape is None else list(shape)} tensor, got {list(t.shape)}")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    _on(t, name, index)
    ld, step = t.stride()
    rows, cols = t.shape
    if step != 1 and cols > 1 and rows > 0:
        raise ValueError(f"{name} must be contiguous in its last dimension")
    if rows > 1:
        if ld < cols:
            raise ValueError(f"{name} must have rows that do not overlap (row pitch {ld}, {cols} columns)")
        return ld
    return max(cols, 1)


def _fp8_pitch(cols: int) -> int:
    return (cols + 15) & ~15


def _fp8_ld(t: torch.Tensor, name: str, index: int, shape=None) -> int:
    """The row pitch of an e4m3 (or INT8) matrix: of a single row, the one that its columns need."""
    ld = _matrix(t, name, index, t.dtype, shape)
    return ld if t.shape[0] > 1 else _fp8_pitch(t.shape[1])


def _scales(t: torch.Tensor, name: str, index: int, groups: int, count: int) -> int:
    return _matrix(t, name, index, torch.float32, (groups, count))


def nq_fp8_quantize(x: torch.Tensor, block_rows: int = 1, rowwise: bool = True, transposed: bool = False):
    """[rows, cols] fp32 / bf16 -> (q, s, qt, st): e4m3 [rows, cols] and its scales, groups first
    ([ceil(cols / 128), rows], or [ceil(cols / 128), ceil(rows / 128)] for block_rows == 128); the same of the transpose
    x^T (groups along the rows of x).  A pair that is not asked for is (None, None)."""
    ld = _matrix(x, "x", x.get_device())
    if x.dtype not in _FLOATS:
        raise ValueError(f"x must be float32 or bfloat16, got {x.dtype}")
    if block_rows not in (1, 128):
        raise ValueError("block_rows must be 1 or 128")
    if not (rowwise or transposed):
        raise ValueError("ask for the matrix (rowwise), its transpose (transposed) or both")
    rows, cols = x.shape
    device, f8, f32 = x.device, torch.float8_e4m3fn, torch.float32
    q = s = qt = st = q_ptr = s_ptr = qt_ptr = st_ptr = None
    ldq, ldqt, lds, ldst = _fp8_pitch(cols), _fp8_pitch(rows), -(-rows // block_rows), -(-cols // block_rows)
    if rowwise:
        q, s = _new(rows, cols, f8, device, ldq), _new((cols + 127) // 128, lds, f32, device)
        q_ptr, s_ptr = q.data_ptr(), s.data_ptr()
    if transposed:
        qt, st = _new(cols, rows, f8, device, ldqt), _new((rows + 127) // 128, ldst, f32, device)
        qt_ptr, st_ptr = qt.data_ptr(), st.data_ptr()
    _check(lib().nq_fp8_quantize(x.data_ptr(), ld, _FLOATS[x.dtype], rows, cols, block_rows, q_ptr, ldq, s_ptr, lds,
                                 qt_ptr, ldqt, st_ptr, ldst, _raw_stream(x)), "nq_fp8_quantize")
    return q, s, qt, st


def nq_fp8_gemm(a: torch.Tensor, sa: torch.Tensor, b: torch.Tensor, sb: torch.Tensor, b_block_rows: int = 128,
                bias: Optional[torch.Tensor] = None, y_dtype: torch.dtype = torch.bfloat16,
                y_out: Optional[torch.Tensor] = None, accumulate: bool = False) -> torch.Tensor:
    """y[m, n] = sum over groups of 128 of sa * sb * (a . b) (+ bias) for e4m3 a [M, K], b [N, K] as nq_fp8_quantize
    writes them: sa [ceil(K / 128), M]; sb [ceil(K / 128), N], or [ceil(K / 128), ceil(N / 128)] for b_block_rows == 128.
    -> y [M, N] fp32 or bf16, or y_out, to which an fp32 product may be added (accumulate)."""
    f8, f32 = torch.float8_e4m3fn, torch.float32
    if a.dtype is not f8 or b.dtype is not f8:
        raise ValueError(f"a and b must be float8_e4m3fn, got {a.dtype} and {b.dtype}")
    if b_block_rows not in (1, 128):
        raise ValueError("b_block_rows must be 1 or 128")
    if a.dim() != 2 or b.dim() != 2 or a.shape[1] != b.shape[1]:
        raise ValueError(f"a and b must be [M, K] and [N, K], got {list(a.shape)} and {list(b.shape)}")
    M, K = a.shape
    N = b.shape[0]
    groups, sb_cols = (K + 127) // 128, -(-N // b_block_rows)
    index = a.get_device()
    if (K & 15 == 0 and a.is_contiguous() and b.is_contiguous() and sa.is_contiguous() and sb.is_contiguous() and sa.dtype is f32
            and sb.dtype is f32 and sa.shape == (groups, M) and sb.shape == (groups, sb_cols)
            and b.get_device() == sa.get_device() == sb.get_device() == index >= 0):
        lda = ldb = K                                    # dense throughout: a call of few microseconds checks no further
        ldsa, ldsb = M, sb_cols
    else:
        lda, ldb = _fp8_ld(a, "a", index), _fp8_ld(b, "b", index)
        ldsa, ldsb = _scales(sa, "sa", index, groups, M), _scales(sb, "sb", index, groups, sb_cols)
    device = a.device
    if y_out is not None:
        y = y_out
        ldy = _matrix(y, "y_out", index, None, (M, N))
    else:
        if accumulate:
            raise ValueError("accumulate needs y_out")
        y = _new(M, N, y_dtype, device)
        ldy = max(N, 1)
    if y.dtype not in _FLOATS:
        raise ValueError(f"the output must be float32 or bfloat16, got {y.dtype}")
    _check(lib().nq_fp8_gemm(a.data_ptr(), lda, sa.data_ptr(), ldsa, b.data_ptr(), ldb, sb.data_ptr(), ldsb, b_block_rows,
                             _vector(bias, "bias", N, index), M, N, K, y.data_ptr(), ldy, _FLOATS[y.dtype], accumulate,
                             _raw_stream(a)), "nq_fp8_gemm")
    return y


# --------------------------------------------------------------------------- block norm
def _vector(t: Optional[torch.Tensor], name: str, cols: int, index: int):
    if t is None:
        return None
    if t.dtype is not torch.float32 or t.dim() != 1 or t.numel() != cols or not t.is_contiguous():
        raise ValueError(f"{name} must be a dense float32 CUDA vector of {cols}")
    _on(t, name, index)
    return t.data_ptr()


def _norm_check(rows, cols, gate, rows_per_gate, post, pre, index):
    if not (0 <= post <= 2 and 0 <= pre <= 2):
        raise ValueError("post and pre are NQ_NORM_NONE, NQ_NORM_RMS or NQ_NORM_LAYER")
    if rows_per_gate < 0:
        raise ValueError("rows_per_gate must not be negative")
    if gate is not None:
        need = -(-rows // rows_per_gate) if rows_per_gate else 1
        if gate.dtype != torch.float32 or not gate.is_contiguous() or gate.shape != (need, cols):
            raise ValueError(f"gate must be a dense float32 CUDA tensor [{need}, {cols}]")
        _on(gate, "gate", index)


def _norm_types(x: torch.Tensor, y: Optional[torch.Tensor], names) -> None:
    if x.dtype not in _FLOATS:
        raise ValueError(f"{names[0]} must be float32 or bfloat16, got {x.dtype}")
    if y is not None and (y.dtype not in _FLOATS or (x.dtype == torch.bfloat16 and y.dtype != torch.bfloat16)):
        raise ValueError(f"({names[0]}, {names[1]}) must be (float32, float32), (float32, bfloat16) or (bfloat16, bfloat16), "
                         f"got ({x.dtype}, {y.dtype})")


def nq_block_norm(x: torch.Tensor, y: Optional[torch.Tensor] = None, *, post: int = NQ_NORM_NONE,
                  post_weight: Optional[torch.Tensor] = None, post_bias: Optional[torch.Tensor] = None,
                  gate: Optional[torch.Tensor] = None, rows_per_gate: int = 0, skip_scale: float = 1.0,
                  branch_scale: float = 1.0, pre: int = NQ_NORM_RMS, pre_weight: Optional[torch.Tensor] = None,
                  pre_bias: Optional[torch.Tensor] = None, eps: float = 1e-6, h_dtype: Optional[torch.dtype] = None,
                  h_scale: float = 1.0, want_r: Optional[bool] = None, r_out: Optional[torch.Tensor] = None):
    """r = skip_scale * x + branch_scale * gate * N_post(y), h = N_pre(r); -> (r, h, hs).

    x, r: the residual stream [rows, cols]; y: the block's output, None for the plain norm of x (then r is returned only
    when want_r).  gate: [1, cols], or one row for each rows_per_gate rows.  h_dtype: float32, bfloat16 (default: y's
    type, without y x's), float8_e4m3fn (hs: its scales, groups first) or int8 (static scale h_scale).  r_out may be x."""
    index = x.get_device()
    ldx = _matrix(x, "x", index)
    _norm_types(x, y, ("x", "y"))
    rows, cols = x.shape
    device = x.device
    _norm_check(rows, cols, gate, rows_per_gate, post, pre, index)
    y_type = x.dtype if y is None else y.dtype
    ldy = 0 if y is None else _matrix(y, "y", index, shape=x.shape)
    r = h = hs = r_ptr = h_ptr = hs_ptr = None
    ldr = ldh = h_code = 0
    if r_out is not None:
        r = r_out
        ldr = _matrix(r, "r_out", index, x.dtype, x.shape)
        r_ptr = r.data_ptr()
    elif want_r or (want_r is None and y is not None):
        r, ldr = _new(rows, cols, x.dtype, device), cols
        r_ptr = r.data_ptr()
    if pre != NQ_NORM_NONE:
        if h_dtype is None:
            h_dtype = y_type
        h_code = _H_TYPES.get(h_dtype)
        if h_code is None:
            raise ValueError(f"h_dtype must be float32, bfloat16, float8_e4m3fn or int8, got {h_dtype}")
        ldh = cols if h_code <= NQ_BF16 else _fp8_pitch(cols)
        h = _new(rows, cols, h_dtype, device, ldh)
        h_ptr = h.data_ptr()
        if h_code == NQ_E4M3:
            hs = _new((cols + 127) // 128, rows, torch.float32, device)
            hs_ptr = hs.data_ptr()
    d = nq_block_norm_desc(rows, cols, ldx, ldy, ldr, ldh, 0, 0, 0, 0, rows_per_gate, _FLOATS[x.dtype], _FLOATS[y_type], h_code,
                           post, pre, skip_scale, branch_scale, eps, h_scale)
    _check(lib().nq_block_norm(ctypes.addressof(d), x.data_ptr(), None if y is None else y.data_ptr(),
                               _vector(post_weight, "post_weight", cols, index), _vector(post_bias, "post_bias", cols, index),
                               None if gate is None else gate.data_ptr(), _vector(pre_weight, "pre_weight", cols, index),
                               _vector(pre_bias, "pre_bias", cols, index), r_ptr, h_ptr, hs_ptr, rows, _raw_stream(x)), "nq_block_norm")
    return r, h, hs


def nq_block_norm_backward_workspace_bytes(desc: nq_block_norm_desc, has_gate: bool) -> int:
    return int(lib().nq_block_norm_backward_workspace_bytes(ctypes.addressof(desc), int(bool(has_gate))))


def nq_block_norm_backward(r: torch.Tensor, y: Optional[torch.Tensor] = None, *, dr: Optional[torch.Tensor] = None,
                           dh: Optional[torch.Tensor] = None, post: int = NQ_NORM_NONE,
                           post_weight: Optional[torch.Tensor] = None, post_bias: Optional[torch.Tensor] = None,
                           gate: Optional[torch.Tensor] = None, rows_per_gate: int = 0, skip_scale: float = 1.0,
                           branch_scale: float = 1.0, pre: int = NQ_NORM_RMS, pre_weight: Optional[torch.Tensor] = None,
                           pre_bias: Optional[torch.Tensor] = None, eps: float = 1e-6,
                           workspace: Optional[torch.Tensor] = None):
    """Gradients of nq_block_norm from the r and y of the forward pass and the gradients dr, dh of its outputs (dh in
    y's type, without y in any that goes with x; one of the two may be None).
    -> (dx, dy, dgate, dpost_weight, dpost_bias, dpre_weight, dpre_bias), None for each input that was absent."""
    index = r.get_device()
    ldr = _matrix(r, "r", index)
    rows, cols = r.shape
    device = r.device
    like = y if y is not None else dh if dh is not None else r
    _norm_types(r, like, ("r", "y" if y is not None else "dh"))
    if (pre == NQ_NORM_NONE) != (dh is None):
        raise ValueError("dh goes with the pre norm: give both or neither")
    if dr is None and dh is None:
        raise ValueError("give dr, dh or both")
    _norm_check(rows, cols, gate, rows_per_gate, post, pre, index)
    y_type = like.dtype
    ldy = 0 if y is None else _matrix(y, "y", index, shape=r.shape)
    lddr = 0 if dr is None else _matrix(dr, "dr", index, r.dtype, r.shape)
    lddh = 0 if dh is None else _matrix(dh, "dh", index, y_type, r.shape)
    d = nq_block_norm_desc(rows, cols, 0, ldy, ldr, 0, cols, cols, lddr, lddh, rows_per_gate, _FLOATS[r.dtype], _FLOATS[y_type], 0,
                           post, pre, skip_scale, branch_scale, eps, 0.0)
    dx = _new(rows, cols, r.dtype, device)
    dy = None if y is None else _new(rows, cols, y_type, device)
    dgate = None if gate is None else torch.empty_like(gate)
    vec = [None if t is None else torch.empty_like(t) for t in (post_weight, post_bias, pre_weight, pre_bias)]
    if workspace is None:
        need = nq_block_norm_backward_workspace_bytes(d, gate is not None)
        workspace = torch.empty_strided((max(need, 16),), (1,), dtype=torch.uint8, device=device)
    else:
        if not workspace.is_contiguous():
            raise ValueError("workspace must be contiguous")
        _on(workspace, "workspace", index)
    ptr = lambda t: None if t is None else t.data_ptr()
    _vector(pre_bias, "pre_bias", cols, index)
    _check(lib().nq_block_norm_backward(
        ctypes.addressof(d), r.data_ptr(), ptr(y), ptr(dr), ptr(dh), _vector(post_weight, "post_weight", cols, index),
        _vector(post_bias, "post_bias", cols, index), ptr(gate), _vector(pre_weight, "pre_weight", cols, index), dx.data_ptr(), ptr(dy),
        ptr(dgate), *map(ptr, vec), workspace.data_ptr(), workspace.numel() * workspace.element_size(),
        _raw_stream(r)), "nq_block_norm_backward")
    return dx, dy, dgate, vec[0], vec[1], vec[2], vec[3]


# --------------------------------------------------------------------------- attention of a served transformer
_CACHE_TYPES = {torch.bfloat16: NQ_BF16, torch.float8_e4m3fn: NQ_E4M3, torch.int8: NQ_I8}


class nq_kv_pages(ctypes.Structure):
    """A paged key-value cache: k, v [pages, kv_heads, page_size, head_dim] bf16, float8_e4m3fn or int8, dense; the latter two with
    fp32 scales ks, vs [pages, kv_heads, page_size].  Holds on to the tensors; made once for a cache, it costs its calls nothing."""
    _fields_ = ([(k, ctypes.c_void_p) for k in ("k", "v", "ks", "vs")] + [("pages", ctypes.c_int64)] +
                [(k, ctypes.c_int32) for k in ("page_size", "kv_heads", "head_dim", "dtype")])

    def __init__(self, k: torch.Tensor, v: torch.Tensor, ks: Optional[torch.Tensor] = None, vs: Optional[torch.Tensor] = None):
        kind, shape, index = k.dtype, k.shape, k.get_device()
        code = _CACHE_TYPES.get(kind)
        if code is None:
            raise ValueError(f"a cache is bfloat16, float8_e4m3fn or int8, got {kind}")
        if len(shape) != 4 or v.shape != shape or v.dtype is not kind:
            raise ValueError(f"k and v must be [pages, kv_heads, page_size, head_dim] of one type, got {list(shape)} {kind} and {list(v.shape)} {v.dtype}")
        if (code == NQ_BF16) != (ks is None) or (code == NQ_BF16) != (vs is None):
            raise ValueError("ks and vs go with a float8_e4m3fn or int8 cache")
        _cache_tensor(k, "k", index)
        _cache_tensor(v, "v", index)
        ks_ptr = vs_ptr = None
        if ks is not None:
            for name, t in (("ks", ks), ("vs", vs)):
                if t.dtype is not torch.float32 or t.shape != shape[:3]:
                    raise ValueError(f"{name} must be float32 {list(shape[:3])}, got {t.dtype} {list(t.shape)}")
                _cache_tensor(t, name, index)
            ks_ptr, vs_ptr = ks.data_ptr(), vs.data_ptr()
        pages, heads, page, dim = shape
        super().__init__(k.data_ptr(), v.data_ptr(), ks_ptr, vs_ptr, pages, page, heads, dim, code)
        self.tensors, self.index = (k, v, ks, vs), index


class _NoGradient(torch.autograd.Function):
    @staticmethod
    def forward(ctx, what, y, *operands):
        ctx.what = what
        ctx.mark_dirty(y)
        return y

    @staticmethod
    def backward(ctx, _):
        raise RuntimeError(f"{ctx.what} has no gradient: call it under torch.no_grad(), or on detached tensors")


def _serving(what: str, y: torch.Tensor, *operands: Optional[torch.Tensor]) -> torch.Tensor:
    """The attention calls have no gradients.  Where one is wanted of an operand, autograd would take their output for a constant: it is tied
    to a node that refuses to be differentiated."""
    if torch.is_grad_enabled():
        for t in operands:
            if t is not None and t.requires_grad:
                return _NoGradient.apply(what, y, *operands)
    return y


def _cache_tensor(t: torch.Tensor, name: str, index: int) -> None:
    if t.get_device() != index or index < 0:
        _on(t, name, index)
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


def _pages_on(cache: nq_kv_pages, index: int) -> int:
    if cache.index != index:
        raise ValueError(f"the cache is on cuda:{cache.index}, the first operand on {'the host' if index < 0 else f'cuda:{index}'}")
    return ctypes.addressof(cache)


def _ints(t: torch.Tensor, name: str, count: int, index: int) -> int:
    if t.dtype is not torch.int32 or t.dim() != 1 or t.shape[0] != count or not t.is_contiguous():
        raise ValueError(f"{name} must be a dense int32 CUDA vector of {count}")
    _on(t, name, index)
    return t.data_ptr()


def _heads(t: torch.Tensor, name: str, index: int, heads: int, dim: int) -> int:
    """Checks [tokens, heads, dim] on the GPU of this index, a token's heads dense; -> its pitch of tokens."""
    if t.dim() != 3 or t.shape[1] != heads or t.shape[2] != dim:
        raise ValueError(f"{name} must be [tokens, {heads}, {dim}], got {list(t.shape)}")
    if t.get_device() != index or index < 0:
        _on(t, name, index)
    if t.is_contiguous():
        return heads * dim
    ld, between, step = t.stride()
    if t.numel() > 0 and ((step != 1 and dim > 1) or (between != dim and heads > 1)):
        raise ValueError(f"{name} must have dense heads in a token (strides {list(t.stride())})")
    if t.shape[0] > 1:
        if ld < heads * dim:
            raise ValueError(f"{name} must have tokens that do not overlap (pitch {ld})")
        return ld
    return heads * dim


def _window(window: int) -> int:
    """A window as the library's int holds it: what passes 32 bits would arrive as another number."""
    if not -(1 << 31) <= window < 1 << 31:
        raise ValueError(f"window must be under 2^31, got {window}")
    return window


def _table(t: torch.Tensor, seqs: int, index: int) -> int:
    if t.dtype is torch.int32 and t.is_contiguous() and t.dim() == 2 and t.shape[0] == seqs and t.get_device() == index >= 0:
        return t.shape[1] or 1
    return _matrix(t, "table", index, torch.int32, (seqs, t.shape[-1]))


def nq_qk_norm_rotate(x: torch.Tensor, angles: Optional[torch.Tensor], positions: Optional[torch.Tensor], *, q_heads: int, kv_heads: int,
                      head_dim: Optional[int] = None, norm: int = NQ_NORM_RMS, q_weight: Optional[torch.Tensor] = None,
                      k_weight: Optional[torch.Tensor] = None, eps: float = 1e-6, neighbours: bool = False,
                      cache: Optional[nq_kv_pages] = None, slots: Optional[torch.Tensor] = None, want_k: Optional[bool] = None,
                      y_dtype: torch.dtype = torch.bfloat16):
    """Rows x [tokens, (q_heads + 2 kv_heads) * head_dim] of a fused projection (queries | keys | values) -> (q [tokens, q_heads,
    head_dim], k [tokens, kv_heads, head_dim] or None): normed for each head, turned by the angles [positions, rotary_dim] (cosines |
    sines) of each token's position.  With a cache and its slots int32 [tokens], keys and values are stored there in the same pass, and
    a dense k comes only when asked for (want_k).  Without one, the values' columns may be missing.  angles None: no rotation."""
    index = x.get_device()
    ldx = _matrix(x, "x", index)
    if x.dtype not in _FLOATS or y_dtype not in _FLOATS:
        raise ValueError(f"x and the output must be float32 or bfloat16, got {x.dtype} and {y_dtype}")
    if q_heads < 0 or kv_heads < 0 or q_heads + kv_heads == 0:
        raise ValueError(f"no heads: q_heads {q_heads}, kv_heads {kv_heads}")
    tokens, width = x.shape
    dim = width // (q_heads + 2 * kv_heads) if head_dim is None else head_dim
    if width != (q_heads + 2 * kv_heads) * dim and (cache is not None or width != (q_heads + kv_heads) * dim):
        raise ValueError(f"x has {width} columns: {q_heads} + 2 * {kv_heads} heads of {dim} are {(q_heads + 2 * kv_heads) * dim}")
    if (cache is None) != (slots is None):
        raise ValueError("cache and slots go together")
    if (angles is None) != (positions is None):
        raise ValueError("angles and positions go together")
    if want_k is None:
        want_k = cache is None
    rows = rotary = 0
    if angles is not None:
        if angles.dtype is not torch.float32 or angles.dim() != 2 or not angles.is_contiguous():
            raise ValueError("angles must be a dense float32 CUDA tensor [positions, rotary_dim]")
        _on(angles, "angles", index)
        rows, rotary = angles.shape
    q = torch.empty_strided((tokens, q_heads, dim), (q_heads * dim, dim, 1), dtype=y_dtype, device=x.device)
    k = torch.empty_strided((tokens, kv_heads, dim), (kv_heads * dim, dim, 1), dtype=y_dtype, device=x.device) if want_k else None
    d = nq_qk_desc(tokens, ldx, q_heads * dim, kv_heads * dim, rows, _FLOATS[x.dtype], _FLOATS[y_dtype], q_heads, kv_heads, dim, rotary, norm, neighbours, eps)
    _check(lib().nq_qk_norm_rotate(ctypes.addressof(d), x.data_ptr(), _vector(q_weight, "q_weight", dim, index), _vector(k_weight, "k_weight", dim, index),
                                   None if angles is None else angles.data_ptr(), None if positions is None else _ints(positions, "positions", tokens, index),
                                   q.data_ptr(), None if k is None else k.data_ptr(), None if cache is None else _pages_on(cache, index),
                                   None if slots is None else _ints(slots, "slots", tokens, index), _raw_stream(x)), "nq_qk_norm_rotate")
    return _serving("nq_qk_norm_rotate", q, x, q_weight), None if k is None else _serving("nq_qk_norm_rotate", k, x, k_weight)


def nq_kv_cache_write(cache: nq_kv_pages, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor) -> None:
    """Stores k, v [tokens, kv_heads, head_dim] (fp32 or bf16) in the slots int32 [tokens], quantised as the cache holds them; a slot
    outside the cache (-1, say) is passed over.  The cache holds values: no gradient leads back through it."""
    index = k.get_device()
    heads, dim = cache.kv_heads, cache.head_dim
    if k.dtype not in _FLOATS or v.dtype is not k.dtype or v.shape != k.shape:
        raise ValueError(f"k and v must be float32 or bfloat16 of one type and shape, got {k.dtype} {list(k.shape)} and {v.dtype} {list(v.shape)}")
    ldk, ldv = _heads(k, "k", index, heads, dim), _heads(v, "v", index, heads, dim)
    tokens = k.shape[0]
    _check(lib().nq_kv_cache_write(_pages_on(cache, index), k.data_ptr(), ldk, v.data_ptr(), ldv, _FLOATS[k.dtype], _ints(slots, "slots", tokens, index),
                                   tokens, _raw_stream(k)), "nq_kv_cache_write")


def nq_kv_cache_read(cache: nq_kv_pages, table: torch.Tensor, starts: torch.Tensor, rows: int, *, y_dtype: torch.dtype = torch.bfloat16,
                     k_out: Optional[torch.Tensor] = None, v_out: Optional[torch.Tensor] = None):
    """The cache's tokens as packed rows -> (k, v) [rows, kv_heads, head_dim]: sequence s, whose pages are table[s] (int32 [sequences,
    columns]), fills rows starts[s] to starts[s + 1] (int32 [sequences + 1]).  Rows of no sequence stay as they were in k_out, v_out."""
    index = table.get_device()
    heads, dim = cache.kv_heads, cache.head_dim
    if (k_out is None) != (v_out is None):
        raise ValueError("give k_out and v_out, or neither")
    if rows < 0:
        raise ValueError("rows must not be negative")
    if k_out is None:
        if y_dtype not in _FLOATS:
            raise ValueError(f"the output must be float32 or bfloat16, got {y_dtype}")
        shape, strides, device = (rows, heads, dim), (heads * dim, dim, 1), table.device
        k_out = torch.empty_strided(shape, strides, dtype=y_dtype, device=device)
        v_out = torch.empty_strided(shape, strides, dtype=y_dtype, device=device)
        ldk = ldv = heads * dim
    else:
        if k_out.dtype not in _FLOATS or v_out.dtype is not k_out.dtype or k_out.shape[0] != rows or v_out.shape[0] != rows:
            raise ValueError(f"k and v must be float32 or bfloat16 with {rows} rows, got {k_out.dtype} {list(k_out.shape)} and {v_out.dtype} {list(v_out.shape)}")
        ldk, ldv = _heads(k_out, "k_out", index, heads, dim), _heads(v_out, "v_out", index, heads, dim)
    seqs = table.shape[0]
    _check(lib().nq_kv_cache_read(_pages_on(cache, index), table.data_ptr(), _table(table, seqs, index), table.shape[-1], _ints(starts, "starts", seqs + 1, index),
                                  seqs, k_out.data_ptr(), ldk, v_out.data_ptr(), ldv, _FLOATS[k_out.dtype], rows, _raw_stream(table)), "nq_kv_cache_read")
    return k_out, v_out


def nq_paged_attention_workspace_bytes(cache: nq_kv_pages, q_heads: int, seqs: int, table_cols: int) -> int:
    return int(lib().nq_paged_attention_workspace_bytes(ctypes.addressof(cache), q_heads, seqs, table_cols))


def nq_paged_attention(q: torch.Tensor, cache: nq_kv_pages, table: torch.Tensor, lengths: torch.Tensor, *, window: int = 0,
                       scale: Optional[float] = None, y_out: Optional[torch.Tensor] = None,
                       workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """One new token a sequence, q bf16 [sequences, q_heads, head_dim], over the first lengths[s] tokens (int32 [sequences]) of the pages
    table[s] (int32 [sequences, columns]), or the last `window` of them -> y like q.  scale: head_dim ** -0.5 where not given.
    A sequence that sees nothing gets zeros."""
    index = q.get_device()
    dim = cache.head_dim
    if q.dtype is not torch.bfloat16:
        raise ValueError(f"q must be bfloat16, got {q.dtype}")
    if q.dim() != 3:
        raise ValueError(f"q must be [sequences, q_heads, {dim}], got {list(q.shape)}")
    seqs, heads = q.shape[:2]
    ldq = _heads(q, "q", index, heads, dim)
    if y_out is None:
        y_out = torch.empty_strided((seqs, heads, dim), (heads * dim, dim, 1), dtype=torch.bfloat16, device=q.device)
        ldy = heads * dim
    else:
        if y_out.dtype is not torch.bfloat16 or y_out.shape != q.shape:
            raise ValueError(f"y_out must be bfloat16 {list(q.shape)}, got {y_out.dtype} {list(y_out.shape)}")
        ldy = _heads(y_out, "y_out", index, heads, dim)
    ld_table, cols = _table(table, seqs, index), table.shape[1]
    pages = _pages_on(cache, index)
    if workspace is None:
        need = lib().nq_paged_attention_workspace_bytes(pages, heads, seqs, cols)
        workspace = torch.empty_strided((max(need, 16),), (1,), dtype=torch.uint8, device=q.device)
    else:
        if not workspace.is_contiguous():
            raise ValueError("workspace must be contiguous")
        _on(workspace, "workspace", index)
    _check(lib().nq_paged_attention(pages, q.data_ptr(), ldq, heads, table.data_ptr(), ld_table, cols, _ints(lengths, "lengths", seqs, index), seqs,
                                    _window(window), dim ** -0.5 if scale is None else scale, y_out.data_ptr(), ldy, workspace.data_ptr(),
                                    workspace.numel() * workspace.element_size(), _raw_stream(q)), "nq_paged_attention")
    return _serving("nq_paged_attention", y_out, q)


def nq_prompt_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, starts_q: torch.Tensor, starts_k: Optional[torch.Tensor] = None, *,
                        causal: bool = True, window: int = 0, scale: Optional[float] = None, y_out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Packed sequences: q bf16 [rows, q_heads, head_dim], k, v bf16 [key rows, kv_heads, head_dim]; sequence s has queries starts_q[s] to
    starts_q[s + 1] and keys starts_k[s] to starts_k[s + 1] (int32 [sequences + 1]; starts_k None: the same) -> y like q.  A causal
    sequence's last query sees all its keys; window: only that many keys up to its own place.  scale: head_dim ** -0.5 where not given.  Rows
    that see nothing are zero; rows of no sequence stay as they were in y_out."""
    index = q.get_device()
    if q.dtype is not torch.bfloat16 or k.dtype is not torch.bfloat16 or v.dtype is not torch.bfloat16:
        raise ValueError(f"q, k and v must be bfloat16, got {q.dtype}, {k.dtype} and {v.dtype}")
    if q.dim() != 3 or k.dim() != 3 or v.shape != k.shape or k.shape[2] != q.shape[2]:
        raise ValueError(f"q, k and v must be [rows, heads, head_dim], k and v alike, got {list(q.shape)}, {list(k.shape)} and {list(v.shape)}")
    rows, heads, dim = q.shape
    kv_heads = k.shape[1]
    ldq, ldk, ldv = _heads(q, "q", index, heads, dim), _heads(k, "k", index, kv_heads, dim), _heads(v, "v", index, kv_heads, dim)
    seqs = starts_q.shape[0] - 1 if starts_q.dim() == 1 else -1
    if seqs < 0:
        raise ValueError("starts_q must be int32 [sequences + 1]")
    if starts_k is None:
        starts_k = starts_q
    if y_out is None:
        y_out = torch.empty_strided((rows, heads, dim), (heads * dim, dim, 1), dtype=torch.bfloat16, device=q.device)
        ldy = heads * dim
    else:
        if y_out.dtype is not torch.bfloat16 or y_out.shape != q.shape:
            raise ValueError(f"y_out must be bfloat16 {list(q.shape)}, got {y_out.dtype} {list(y_out.shape)}")
        ldy = _heads(y_out, "y_out", index, heads, dim)
    d = nq_prompt_desc(seqs, rows, k.shape[0], ldq, ldk, ldv, ldy, heads, kv_heads, dim, causal, _window(window), dim ** -0.5 if scale is None else scale)
    _check(lib().nq_prompt_attention(ctypes.addressof(d), q.data_ptr(), k.data_ptr(), v.data_ptr(), _ints(starts_q, "starts_q", seqs + 1, index),
                                     _ints(starts_k, "starts_k", seqs + 1, index), y_out.data_ptr(), _raw_stream(q)), "nq_prompt_attention")
    return _serving("nq_prompt_attention", y_out, q, k, v)


def nq_i8_mma_ceiling(stage_iters: int) -> float:
    """Enqueues one launch of the MMA-issue-only kernel on the current stream; returns its integer operations."""
    ops = ctypes.c_double(0.0)
    _check(lib().nq_i8_mma_ceiling(_i64(stage_iters), ctypes.byref(ops), _stream()), "nq_i8_mma_ceiling")
    return float(ops.value)


def nq_device_status() -> int:
    """Synchronises the current stream; raises NqError(NQ_ERR_TIMEOUT) if a bounded device wait expired."""
    where = ctypes.c_int(0)
    st = lib().nq_device_status(_stream(), ctypes.byref(where))
    if st != NQ_OK:
        raise NqError(st, f"nq_device_status (wait code {where.value})")
    return 0
