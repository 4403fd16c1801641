"""The attention half of a transformer, served: prompts of different lengths packed behind one another, then a token at a time, over a
paged key-value cache in bf16, e4m3 or INT8.  Every step of its arithmetic runs in the kernels behind ``include/nq.h``.

  prompt   block norm to e4m3 -> fused projection (nq_fp8_gemm) -> heads normed and rotated, keys and values to the cache
           (nq_qk_norm_rotate) -> nq_prompt_attention, over what nq_kv_cache_read brings back where the sequences have a prefix -> projection
  token    the same, with nq_paged_attention over the cache

``python -m paper_2506_17870_b200.attention`` serves a small stack: prompts, then tokens, against the same tokens as one prompt.
"""
from __future__ import annotations

from typing import List, NamedTuple, Optional, Sequence

import numpy as np
import torch

from . import binding as nq
from .fp8_block import MlpBlock, MlpStack, ServedBlock


def rotary_angles(positions: int, rotary_dim: int, base: float = 10000.0, device="cuda") -> torch.Tensor:
    """The table of nq_qk_norm_rotate: [positions, rotary_dim] fp32, cosines | sines of position * base^(-2 i / rotary_dim), computed in 64 bits."""
    at = torch.arange(positions, dtype=torch.float64, device=device)[:, None] * base ** (
        -torch.arange(0, rotary_dim, 2, dtype=torch.float64, device=device) / max(rotary_dim, 1))
    return torch.cat([at.cos(), at.sin()], 1).float()


class Batch(NamedTuple):
    """New tokens of some sequences, packed: where they go, and where the sequences' tokens are."""
    positions: torch.Tensor            # int32 [tokens]
    slots: torch.Tensor                # int32 [tokens]
    starts: torch.Tensor               # int32 [sequences + 1]: the new tokens
    starts_all: torch.Tensor           # int32 [sequences + 1]: all tokens, the new ones included
    table: torch.Tensor                # int32 [sequences, columns]: pages
    lengths: torch.Tensor              # int32 [sequences], the new tokens included
    rows_all: int
    single: bool                       # one new token each
    fresh: bool                        # nobody has earlier tokens
    longest: int = 0                   # tokens of the longest sequence, the new ones included


class PageTable:
    """Which pages of a cache (or of the caches of several layers) each sequence holds.  Kept on the host; extend() hands out what a
    pass over new tokens needs on the device.  positions: how many tokens a sequence may have (None: as many as there are pages for).  Where they are given, a batch's table has
    columns for all of them, so that a captured pass over its tensors follows sequences into new pages."""

    def __init__(self, pages: int, page_size: int, device="cuda", positions: Optional[int] = None):
        if pages < 0 or page_size < 1:
            raise ValueError(f"{pages} pages of {page_size} tokens")
        if positions is not None and positions < 0:
            raise ValueError(f"{positions} positions")
        self.page_size, self.device, self.positions = page_size, device, positions
        self.columns = None if positions is None else max(1, min(pages, -(-positions // page_size)))
        self._free = list(range(pages - 1, -1, -1))
        self._held: dict = {}                                  # sequence -> its pages
        self._length: dict = {}
        self._next = 0

    @property
    def free_pages(self) -> int:
        return len(self._free)

    def length(self, sequence: int) -> int:
        return self._length[sequence]

    def add(self) -> int:
        """A new, empty sequence; -> its number."""
        number, self._next = self._next, self._next + 1
        self._held[number], self._length[number] = [], 0
        return number

    def drop(self, sequence: int) -> None:
        """Ends a sequence; its pages are free for others."""
        self._free += reversed(self._held.pop(sequence))
        del self._length[sequence]

    def extend(self, sequences: Sequence[int], counts: Sequence[int]) -> Batch:
        """Room for counts[i] new tokens of each sequence.  Raises before anything changes when there are not enough pages or positions."""
        if len(sequences) != len(counts) or len(set(sequences)) != len(sequences):
            raise ValueError("one count for each sequence, and each sequence once")
        if any(c < 0 for c in counts):
            raise ValueError("counts must not be negative")
        ps = self.page_size
        longest = max((self._length[s] + c for s, c in zip(sequences, counts)), default=0)
        if self.positions is not None and longest > self.positions:
            raise RuntimeError(f"{longest} tokens of a sequence, there are {self.positions} positions")
        need = [-(-(self._length[s] + c) // ps) - len(self._held[s]) for s, c in zip(sequences, counts)]
        if sum(need) > len(self._free):
            raise RuntimeError(f"{sum(need)} pages needed, {len(self._free)} free")
        positions: List[int] = []
        slots: List[int] = []
        starts, starts_all, lengths = [0], [0], []
        fresh = True
        for s, c, n in zip(sequences, counts, need):
            self._held[s] += [self._free.pop() for _ in range(n)]
            at = self._length[s]
            fresh = fresh and at == 0
            for t in range(at, at + c):
                positions.append(t)
                slots.append(self._held[s][t // ps] * ps + t % ps)
            self._length[s] = at + c
            lengths.append(at + c)
            starts.append(starts[-1] + c)
            starts_all.append(starts_all[-1] + at + c)
        columns = self.columns or max([1] + [len(self._held[s]) for s in sequences])
        table = np.full((len(sequences), columns), -1, np.int32)
        for row, s in zip(table, sequences):
            row[:len(self._held[s])] = self._held[s]
        ints = lambda v, *shape: torch.tensor(v, dtype=torch.int32).reshape(*shape).to(self.device)
        return Batch(ints(positions, -1), ints(slots, -1), ints(starts, -1), ints(starts_all, -1), torch.from_numpy(table).to(self.device), ints(lengths, -1),
                     starts_all[-1], all(c == 1 for c in counts), fresh, longest)


class AttentionBlock(ServedBlock):
    """norm -> fused projection -> heads normed and rotated -> attention -> projection, for serving; its output meets the stream as an
    MlpBlock's does.  Holds the cache of its layer (empty until cache() makes it)."""
    linears = ("qkv", "out")

    def __init__(self, width: int, q_heads: int, kv_heads: int, head_dim: int, device="cuda"):
        super().__init__()
        if q_heads % kv_heads:
            raise ValueError(f"{q_heads} query heads over {kv_heads} key heads")
        self.q_heads, self.kv_heads, self.head_dim = q_heads, kv_heads, head_dim
        new = lambda *shape: torch.nn.Parameter(torch.ones(*shape, device=device), requires_grad=False)
        self.pre_weight, self.post_weight, self.gate = new(width), new(width), new(1, width)
        self.q_weight, self.k_weight = new(head_dim), new(head_dim)
        self.qkv, self.out = new((q_heads + 2 * kv_heads) * head_dim, width), new(width, q_heads * head_dim)
        self.gate.fill_(0.5)
        self.qkv.normal_(std=width ** -0.5)
        self.out.normal_(std=(q_heads * head_dim) ** -0.5)
        self.pages: Optional[nq.nq_kv_pages] = None

    def cache(self, pages: int, page_size: int, dtype: torch.dtype = torch.float8_e4m3fn) -> None:
        """Makes the layer's cache, empty."""
        shape = (pages, self.kv_heads, page_size, self.head_dim)
        device = self.qkv.device
        codes = lambda: torch.zeros(shape, dtype=torch.bfloat16 if dtype is torch.bfloat16 else torch.uint8, device=device).view(dtype)
        scales = lambda: None if dtype is torch.bfloat16 else torch.zeros(shape[:3], device=device)
        self.pages = nq.nq_kv_pages(codes(), codes(), scales(), scales())

    def __getstate__(self):
        return {**super().__getstate__(), "pages": None}       # a copy has no cache

    @torch.no_grad()
    def serve(self, h: torch.Tensor, hs: torch.Tensor, batch: Batch, angles: torch.Tensor) -> torch.Tensor:
        if batch.longest > angles.shape[0]:                    # their keys would be NaN, and stay in the cache
            raise ValueError(f"{batch.longest} tokens of a sequence, angles of {angles.shape[0]} positions")
        qkv, out = self._laid_out()
        if self.pages is None:
            raise RuntimeError("the layer has no cache: call cache()")
        x = nq.nq_fp8_gemm(h, hs, qkv.q, qkv.s)
        dense = batch.fresh and not batch.single               # the new tokens are all there is: no need to read them back
        q, k = nq.nq_qk_norm_rotate(x, angles, batch.positions, q_heads=self.q_heads, kv_heads=self.kv_heads, q_weight=self.q_weight,
                                    k_weight=self.k_weight, cache=self.pages, slots=batch.slots, want_k=dense)
        if batch.single:
            y = nq.nq_paged_attention(q, self.pages, batch.table, batch.lengths)
        elif dense:
            v = x.unflatten(1, (-1, self.head_dim))[:, self.q_heads + self.kv_heads:]
            y = nq.nq_prompt_attention(q, k, v, batch.starts)
        else:
            k, v = nq.nq_kv_cache_read(self.pages, batch.table, batch.starts_all, batch.rows_all)
            y = nq.nq_prompt_attention(q, k, v, batch.starts, batch.starts_all)
        q8, s8, _, _ = nq.nq_fp8_quantize(y.flatten(1))
        return nq.nq_fp8_gemm(q8, s8, out.q, out.s)


class _Mlp(MlpBlock):
    def serve(self, h, hs, *_):
        return super().serve(h, hs)


class DecoderStack(MlpStack):
    """Attention and MLP blocks in turn, served."""

    def __init__(self, layers: int, width: int, hidden: int, q_heads: int, kv_heads: int, head_dim: int, positions: int, skip_scale: float = 1.0,
                 branch_scale: float = 1.0, device="cuda"):
        super().__init__(0, width, hidden, skip_scale, branch_scale, device)
        for _ in range(layers):
            self.blocks.append(AttentionBlock(width, q_heads, kv_heads, head_dim, device))
            self.blocks.append(_Mlp(width, hidden, device))
        self.angles = rotary_angles(positions, head_dim, device=device)

    def _apply(self, *args, **kwargs):
        super()._apply(*args, **kwargs)
        device = self.final_weight.device                      # the angles go where the weights go, and stay fp32
        if self.angles.is_meta and device.type != "meta":
            self.angles = rotary_angles(*self.angles.shape, device=device)
        self.angles = self.angles.to(device)
        return self

    def forward(self, x):
        raise RuntimeError("a DecoderStack is for serving: call serve()")

    def cache(self, pages: int, page_size: int, dtype: torch.dtype = torch.float8_e4m3fn) -> PageTable:
        """Makes each layer's cache; -> who holds which of their pages."""
        for b in self.blocks:
            if isinstance(b, AttentionBlock):
                b.cache(pages, page_size, dtype)
        return PageTable(pages, page_size, self.final_weight.device, self.angles.shape[0])

    def serve(self, x: torch.Tensor, batch: Batch) -> torch.Tensor:
        """New tokens' stream [tokens, width], packed as the batch says -> the final norm's output."""
        return super().serve(x, batch, self.angles)


def main(layers: int = 2, width: int = 512, hidden: int = 1536, q_heads: int = 8, kv_heads: int = 2, head_dim: int = 64) -> float:
    """Serves three prompts, then eight tokens each, and the whole sequences again as prompts; -> how far the two are apart."""
    torch.manual_seed(0)
    stack = DecoderStack(layers, width, hidden, q_heads, kv_heads, head_dim, positions=2048)
    stack.freeze()
    lengths, more = [700, 33, 256], 8
    x = [torch.randn(n + more, width, device="cuda", dtype=torch.bfloat16) for n in lengths]
    table = stack.cache(pages=160, page_size=16)
    ids = [table.add() for _ in lengths]
    stack.serve(torch.cat([v[:n] for v, n in zip(x, lengths)]), table.extend(ids, lengths))
    out = [stack.serve(torch.stack([v[n + t] for v, n in zip(x, lengths)]), table.extend(ids, [1] * len(ids))) for t in range(more)]
    step = torch.stack(out, 1).float()
    for i in ids:
        table.drop(i)
    ids = [table.add() for _ in lengths]
    whole = stack.serve(torch.cat(x), table.extend(ids, [len(v) for v in x])).float().split([len(v) for v in x])
    whole = torch.stack([v[-more:] for v in whole])
    nq.nq_device_status()
    far = float((step - whole).norm() / whole.norm())
    print(f"{len(lengths)} prompts, then {more} tokens each over an e4m3 cache: {far:.4f} of the norm from the same tokens as one prompt")
    return far


if __name__ == "__main__":
    main()
