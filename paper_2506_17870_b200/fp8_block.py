"""The linear half of a transformer in e4m3, trained and served: the block-scaled product, its quantiser and the block
norm, strung together as a user would.  Every step of their arithmetic runs in the kernels behind ``include/nq.h``; torch
supplies the memory, the autograd graph, the activation between the two linears and the optimiser.

  training   block norm (bf16 out) -> quantised both ways -> product; backward: gradient quantised both ways -> input
             gradient (blocks of W^T), weight gradient (both transposes, fp32), block norm backward
  serving    block norm straight to e4m3 -> product -> activation -> quantised -> product, for one token or many
  INT8       block norm straight to INT8 (static scale) -> nq_gemm_nested on the two stored parts of a nested weight

``python -m paper_2506_17870_b200.fp8_block`` trains a small stack on synthetic data and serves it.
"""
from __future__ import annotations

from typing import List, NamedTuple, Optional, Tuple

import torch

from . import binding as nq


class Fp8Weight(NamedTuple):
    """A weight [out, in] in blocks of 128 x 128, as it is and transposed; laid out once, kept while it does not change."""
    q: torch.Tensor
    s: torch.Tensor
    qt: torch.Tensor
    st: torch.Tensor


def quantize_weight(w: torch.Tensor) -> Fp8Weight:
    return Fp8Weight(*nq.nq_fp8_quantize(w, block_rows=128, transposed=True))


class _Refusal(torch.autograd.Function):
    @staticmethod
    def forward(ctx, anchor, grad):
        return grad.view_as(grad)

    @staticmethod
    def backward(ctx, _):
        raise RuntimeError("the gradients of fp8_linear and block_norm cannot be differentiated again")


def _first_order(*grads):
    """Gradients out of kernels, of which autograd knows no more than their values.  Where they become part of a graph
    (create_graph) it would take them for constants: they are tied to a node that refuses to be differentiated."""
    if not torch.is_grad_enabled():
        return grads
    anchor = torch.zeros((), requires_grad=True)
    return tuple(None if g is None else _Refusal.apply(anchor, g) for g in grads)


class _Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias):
        q, s, qt, st = nq.nq_fp8_quantize(x, transposed=True)
        w = quantize_weight(weight)
        ctx.save_for_backward(qt, st, w.qt, w.st)
        ctx.has_bias = bias is not None
        return nq.nq_fp8_gemm(q, s, w.q, w.s, bias=bias, y_dtype=x.dtype)

    @staticmethod
    def backward(ctx, dy):
        xt, sxt, wt, swt = ctx.saved_tensors
        d, sd, dt, sdt = nq.nq_fp8_quantize(dy.contiguous(), transposed=True)
        dx = nq.nq_fp8_gemm(d, sd, wt, swt, y_dtype=dy.dtype)
        dw = nq.nq_fp8_gemm(dt, sdt, xt, sxt, b_block_rows=1, y_dtype=torch.float32)
        return *_first_order(dx, dw), dy.float().sum(0) if ctx.has_bias else None


def fp8_linear(x: torch.Tensor, weight: torch.Tensor, bias: Optional[torch.Tensor] = None) -> torch.Tensor:
    """x [tokens, in] fp32 or bf16, weight [out, in] fp32 -> x W^T + bias in x's type, with gradients."""
    return _Linear.apply(x, weight, bias)


class _BlockNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, y, post_weight, post_bias, gate, pre_weight, pre_bias, how, output):
        r, h, _ = nq.nq_block_norm(x, y, post_weight=post_weight, post_bias=post_bias, gate=gate, pre_weight=pre_weight, pre_bias=pre_bias,
                                   want_r=True, **how, **output)
        ctx.how = how
        ctx.save_for_backward(r, y, post_weight, post_bias, gate, pre_weight, pre_bias)
        return r, h

    @staticmethod
    def backward(ctx, dr, dh):
        r, y, post_weight, post_bias, gate, pre_weight, pre_bias = ctx.saved_tensors
        if dh is not None:                                     # (no pre norm, no h)
            # it comes in h's type, the kernel takes it in the branch's; alone, a bf16 stream goes with bf16 only
            kind = y.dtype if y is not None else r.dtype if r.dtype == torch.bfloat16 else dh.dtype
            dh = dh.contiguous().to(kind)
        dx, dy, dgate, dpost_weight, dpost_bias, dpre_weight, dpre_bias = nq.nq_block_norm_backward(
            r, y, dr=dr.contiguous(), dh=dh, post_weight=post_weight, post_bias=post_bias, gate=gate, pre_weight=pre_weight,
            pre_bias=pre_bias, **ctx.how)
        return *_first_order(dx, dy, dpost_weight, dpost_bias, dgate, dpre_weight, dpre_bias), None, None


def block_norm(x: torch.Tensor, y: Optional[torch.Tensor], post_weight: Optional[torch.Tensor], gate: Optional[torch.Tensor],
               pre_weight: Optional[torch.Tensor], *, post_bias: Optional[torch.Tensor] = None, pre_bias: Optional[torch.Tensor] = None,
               post: Optional[int] = None, pre: int = nq.NQ_NORM_RMS, rows_per_gate: int = 0, skip_scale: float = 1.0,
               branch_scale: float = 1.0, eps: float = 1e-6, h_dtype: Optional[torch.dtype] = None,
               h_scale: float = 1.0) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """(r, h) of nq_block_norm, with gradients; without y, r = skip_scale * x and there is no post norm; without a pre norm
    (pre=NQ_NORM_NONE) h is None.  The gradient of an h whose type is not y's (h_dtype) is rounded to y's.  An INT8 h (with its
    h_scale) has none and comes only where no gradient is wanted; e4m3 codes come with their scales, from nq_block_norm."""
    how = dict(post=(nq.NQ_NORM_NONE if y is None else nq.NQ_NORM_RMS) if post is None else post, pre=pre, rows_per_gate=rows_per_gate,
               skip_scale=skip_scale, branch_scale=branch_scale, eps=eps)
    tensors = (x, y, post_weight, post_bias, gate, pre_weight, pre_bias)
    if h_dtype is torch.float8_e4m3fn:
        raise ValueError("e4m3 output has scales: call nq_block_norm")
    if h_dtype is torch.int8 and torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in tensors):
        raise ValueError("INT8 output has no gradient: call block_norm under no_grad, or nq_block_norm")
    return _BlockNorm.apply(*tensors, how, dict(h_dtype=h_dtype, h_scale=h_scale))


class MlpBlock(torch.nn.Module):
    """norm -> up -> activation -> down; its output meets the stream in the next block's (or the final) norm, which
    applies this block's post norm, gate and residual scale."""

    def __init__(self, width: int, hidden: int, device="cuda"):
        super().__init__()
        new = lambda *shape: torch.nn.Parameter(torch.empty(*shape, device=device))
        self.pre_weight, self.post_weight, self.gate = new(width), new(width), new(1, width)
        self.up, self.down, self.up_bias = new(hidden, width), new(width, hidden), new(hidden)
        with torch.no_grad():
            self.pre_weight.fill_(1.0)
            self.post_weight.fill_(1.0)
            self.gate.fill_(0.5)
            self.up_bias.zero_()
            self.up.normal_(std=width ** -0.5)
            self.down.normal_(std=hidden ** -0.5)
        self.served: Optional[Tuple[Fp8Weight, Fp8Weight]] = None
        self._served_from = None                               # what up and down were when they were laid out

    def forward(self, h: torch.Tensor) -> torch.Tensor:
        y = fp8_linear(torch.nn.functional.gelu(fp8_linear(h, self.up, self.up_bias)), self.down)
        if y.requires_grad and (self.up.requires_grad or self.down.requires_grad):
            y.register_hook(self._backward_came)
        return y

    def _backward_came(self, _) -> None:
        self._served_from = None                               # a fused optimiser's step is not counted as a write

    def _weights(self):
        """The two weights, where they lie and how often they were written (not counting writes through .data)."""
        return [(w, w.data_ptr(), 0 if w.is_inference() else w._version) for w in (self.up, self.down)]

    def _served_as_they_are(self) -> bool:
        return self._served_from is not None and all(a is b and rest == now for (a, *rest), (b, *now) in zip(self._served_from, self._weights()))

    # a copy of a block has weights of its own
    def __getstate__(self):
        return {**self.__dict__, "_served_from": self._served_as_they_are()}

    def __setstate__(self, state):
        super().__setstate__(state)
        self._served_from = self._weights() if state.get("_served_from") else None
        if self._served_from is None:
            self.served = None

    @torch.no_grad()
    def freeze(self) -> None:
        """Lays the weights out for serving; to be called again after a backward pass or a change of the weights.  (Not noticed
        by serve(): writes through .data, and a fused optimiser's step on gradients from before this call.)"""
        self.served, self._served_from = (quantize_weight(self.up), quantize_weight(self.down)), self._weights()

    @torch.no_grad()
    def serve(self, h: torch.Tensor, hs: torch.Tensor) -> torch.Tensor:
        if not self._served_as_they_are():
            raise RuntimeError("the weights were not laid out for serving, or were trained or changed since: call freeze()")
        up, down = self.served
        a = torch.nn.functional.gelu(nq.nq_fp8_gemm(h, hs, up.q, up.s, bias=self.up_bias))
        q, s, _, _ = nq.nq_fp8_quantize(a)
        return nq.nq_fp8_gemm(q, s, down.q, down.s)


class MlpStack(torch.nn.Module):
    def __init__(self, blocks: int, width: int, hidden: int, skip_scale: float = 1.0, branch_scale: float = 1.0, device="cuda"):
        super().__init__()
        self.blocks = torch.nn.ModuleList(MlpBlock(width, hidden, device) for _ in range(blocks))
        self.final_weight = torch.nn.Parameter(torch.ones(width, device=device))
        self.how = dict(skip_scale=skip_scale, branch_scale=branch_scale)

    def _between(self, i: int):
        """What stands before block i: the post norm and gate of the block before it, and the pre norm of this one."""
        last = self.blocks[i - 1] if i else None
        pre = self.blocks[i].pre_weight if i < len(self.blocks) else self.final_weight
        return (last.post_weight, last.gate, pre, self.how) if i else (None, None, pre, {})

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        y = None
        for i in range(len(self.blocks) + 1):
            post, gate, pre, how = self._between(i)
            x, h = block_norm(x, y, post, gate, pre, **how)
            if i < len(self.blocks):
                y = self.blocks[i](h)
        return h

    def freeze(self) -> None:
        for b in self.blocks:
            b.freeze()

    @torch.no_grad()
    def serve(self, x: torch.Tensor) -> torch.Tensor:
        """The same for one token or many, with the norms' outputs as e4m3 operands."""
        y = None
        for i in range(len(self.blocks) + 1):
            post, gate, pre, how = self._between(i)
            kind = nq.NQ_NORM_NONE if y is None else nq.NQ_NORM_RMS
            final = i == len(self.blocks)
            r, h, hs = nq.nq_block_norm(x, y, post=kind, post_weight=post, gate=gate, pre_weight=pre,
                                        h_dtype=torch.bfloat16 if final else torch.float8_e4m3fn, **how)
            x = x if r is None else r
            if not final:
                y = self.blocks[i].serve(h, hs)
        return h


class NestedLinear:
    """A linear on a nested INT8 weight behind a block norm whose output is INT8: what the norm hands over is the
    activation operand of nq_gemm_nested (full-bit) or nq_gemm_part (part-bit, w_high alone)."""

    def __init__(self, w_int: torch.Tensor, w_scale: torch.Tensor, h_bits: int, act_scale: float, mask: torch.Tensor):
        self.rows, self.h_bits, self.w_scale, self.act_scale = w_int.shape[0], h_bits, w_scale, act_scale
        self.high, self.low = nq.nq_decompose(w_int, mask, 8, h_bits, True)

    def __call__(self, x: torch.Tensor, pre_weight: torch.Tensor, pre_bias: Optional[torch.Tensor], part_bit: bool = False) -> torch.Tensor:
        _, h, _ = nq.nq_block_norm(x, None, pre=nq.NQ_NORM_LAYER, pre_weight=pre_weight, pre_bias=pre_bias, h_dtype=torch.int8,
                                   h_scale=self.act_scale)
        if part_bit:
            return nq.nq_gemm_part(h, self.high, self.rows, 8, self.h_bits, self.w_scale, self.act_scale)[1]
        return nq.nq_gemm_nested(h, self.high, self.low, self.rows, 8, self.h_bits, self.w_scale, self.act_scale)[1]


def main(steps: int = 60, tokens: int = 2048, width: int = 512, hidden: int = 2048, blocks: int = 3) -> List[float]:
    """Fits a stack to a fixed random stack's outputs; prints the loss, then serves one token and the batch."""
    torch.manual_seed(0)
    teacher, student = MlpStack(blocks, width, hidden), MlpStack(blocks, width, hidden)
    optimiser = torch.optim.AdamW(student.parameters(), lr=2e-3)
    losses = []
    for step in range(steps):
        x = torch.randn(tokens, width, device="cuda", dtype=torch.bfloat16)
        with torch.no_grad():
            want = teacher(x)
        loss = (student(x).float() - want.float()).square().mean()
        optimiser.zero_grad(set_to_none=True)
        loss.backward()
        optimiser.step()
        losses.append(float(loss.detach()))
        if step % 10 == 0 or step == steps - 1:
            print(f"step {step:3d}  loss {losses[-1]:.5f}")
    student.freeze()
    with torch.no_grad():
        trained = student(x).float()
    many, one = student.serve(x).float(), student.serve(x[:1]).float()
    print(f"served against trained forward: {float((many - trained).norm() / trained.norm()):.4f} of the norm; "
          f"one token against the batch: {float((one - many[:1]).norm() / one.norm()):.4f}")
    return losses


if __name__ == "__main__":
    main()
