"""The decoder block around the expert FFN, for decoding with drafted tokens.

QuantLinear   a 4-bit weight matrix in device memory and its product
PagedCache    one layer's paged key/value cache and the calls over it
DecoderBlock  norm -> q/k/v -> rotate and store -> attend -> project -> add and
              norm -> MoELayer -> add and norm of the next block, one C call a step
tree_mask     the mask words of a tree of drafts from its parents

The classes own buffers and marshal; every step runs in the library's kernels.
"""
from __future__ import annotations

import math
from typing import Dict, Optional, Sequence

import numpy as np
import torch

from . import api
from ._lib import TYPE_BF16, TYPE_FP16, CacheDesc, MoEError

_TYPE16 = {torch.bfloat16: TYPE_BF16, torch.float16: TYPE_FP16}


def tree_mask(parents: Sequence[Sequence[int]], device="cuda") -> torch.Tensor:
    """Mask words int64 [tokens][ceil(most drafts / 64)] of drafted trees: parents[b][i] is
    the index, below i, of the draft that draft i of sequence b continues, -1 for one that
    continues the cached text.  Bit m of a row: the draft itself or an ancestor of it."""
    width = max([1] + [(len(p) + 63) // 64 for p in parents])
    words = np.zeros((sum(len(p) for p in parents), width), np.uint64)
    n = 0
    for par in parents:
        for i, p in enumerate(par):
            if not -1 <= p < i:
                raise MoEError("draft %d continues %d: a parent comes before its draft" % (i, p))
            if p >= 0:
                words[n + i] = words[n + p]
            words[n + i, i // 64] |= np.uint64(1 << (i % 64))
        n += len(par)
    return torch.from_numpy(words.view(np.int64)).to(device)


class QuantLinear:
    """A [R][K] weight matrix at 4 bits (packed by moe_quant_pack) and its product."""

    def __init__(self, w: torch.Tensor, group: int = 128, bias: Optional[torch.Tensor] = None):
        if w.dtype != torch.float32 or w.dim() != 2 or not w.is_cuda or w.stride(1) != 1:
            raise MoEError("w must be a float32 device matrix")
        self.R, self.K = w.shape
        self.bias = bias
        if group not in (64, 128) or self.K % group:
            raise MoEError("K = %d is not a multiple of the group %d" % (self.K, group))
        ld = self.K // 8 + 16   # padded, so that rows spread over the memory channels
        self.codes = torch.empty(self.R, ld, dtype=torch.int32, device=w.device)
        self.sz = torch.empty(self.K // group, self.R, dtype=torch.int32, device=w.device)
        status = torch.zeros(1, dtype=torch.int32, device=w.device)
        api.moe_quant_pack(w, 4, group, self.codes, self.sz, ld_codes=ld, sz_row_stride=1, sz_group_stride=self.R,
                           status=status)
        if int(status.item()) != 0:
            raise MoEError("moe_quant_pack reported status %d" % int(status.item()))

    def __call__(self, x: torch.Tensor, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """x [T][K] bf16 or fp16 -> [T][R] (a new tensor of x's type unless `out` is given)."""
        if out is None:
            out = api._empty((x.shape[0], self.R), x.dtype, x.device, stream)
        api.moe_quant_linear(x, self.codes, self.sz, out, bias=self.bias, stream=stream)
        return out


class PagedCache:
    """One layer's key/value cache over the caller's tensors.

    k      [pages][heads][page_size][head_dim], v [pages][heads][head_dim][page_size]
           (transposed inside the page), bfloat16 or float16
    table  int32 [sequences][max_pages], lens int32 [sequences] (cached tokens)

    The attention's workspace is kept per stream and grows with the calls (it at least
    doubles).  A call that is being captured works in memory of its graph's own pool
    instead.  So calls on different streams are independent, and so are replays of
    graphs that share no pool, except that writers of the same pages must be ordered
    by the caller, as for any device memory.
    """

    def __init__(self, k: torch.Tensor, v: torch.Tensor, table: torch.Tensor, lens: torch.Tensor,
                 status: Optional[torch.Tensor] = None):
        if k.dim() != 4 or k.dtype not in _TYPE16 or v.dtype != k.dtype:
            raise MoEError("k and v must be 4-dimensional bfloat16 or float16 tensors of one type")
        n_pages, heads, page, D = k.shape
        if tuple(v.shape) != (n_pages, heads, D, page):
            raise MoEError("v must be [pages][heads][head_dim][page_size]: %s" % ((n_pages, heads, D, page),))
        if not (k.is_cuda and v.is_cuda and k.is_contiguous() and v.is_contiguous()):
            raise MoEError("k and v must be contiguous device tensors")
        self.k, self.v, self.table, self.lens = k, v, table, lens
        self.status = torch.zeros(1, dtype=torch.int32, device=k.device) if status is None else status
        d = CacheDesc()
        d.k, d.v = k.data_ptr(), v.data_ptr()
        d.n_pages, d.n_heads, d.page_size, d.head_dim, d.type = n_pages, heads, page, D, _TYPE16[k.dtype]
        self.desc = d
        self._ws: Dict[int, torch.Tensor] = {}
        self._need: Dict[tuple, int] = {}

    @classmethod
    def create(cls, n_seqs: int, max_len: int, n_heads: int, head_dim: int, page_size: int = 64,
               dtype: torch.dtype = torch.bfloat16, device="cuda") -> "PagedCache":
        """An empty cache with pages of its own for every sequence's max_len tokens."""
        per = (max_len + page_size - 1) // page_size
        k = torch.empty(n_seqs * per, n_heads, page_size, head_dim, dtype=dtype, device=device)
        v = torch.empty(n_seqs * per, n_heads, head_dim, page_size, dtype=dtype, device=device)
        table = torch.arange(n_seqs * per, dtype=torch.int32, device=device).view(n_seqs, per)
        return cls(k, v, table, torch.zeros(n_seqs, dtype=torch.int32, device=device))

    def status_value(self) -> int:
        """0, or MOE_ERR_SLOT once a page, length, position or draft index was out of range;
        reads it back."""
        return int(self.status.item())

    def append(self, q: Optional[torch.Tensor], k: torch.Tensor, v: torch.Tensor, new_off: torch.Tensor,
               max_new: int, positions: Optional[torch.Tensor] = None, cos: Optional[torch.Tensor] = None,
               sin: Optional[torch.Tensor] = None, interleaved: bool = False,
               q_out: Optional[torch.Tensor] = None, stream=None) -> Optional[torch.Tensor]:
        """Rotate q and k, store k and v of the new tokens; returns the rotated q."""
        if q is not None and q_out is None:
            q_out = api._empty(q.shape, q.dtype, q.device, stream)
        api.moe_cache_append(self.desc, self.table, self.lens, new_off, max_new, q, k, v, q_out, positions, cos,
                             sin, interleaved, self.status, stream)
        return q_out

    def _workspace(self, n_q_heads: int, max_new: int, max_len: int, stream) -> Optional[torch.Tensor]:
        key = (n_q_heads, self.lens.shape[0], max_new, max_len)
        need = self._need.get(key)
        if need is None:
            if len(self._need) > 4096:
                self._need.clear()
            need = self._need[key] = api.moe_tree_attention_plan(self.desc, *key)[1]
        if need == 0:
            return None
        if api._capturing(stream):   # the stream of a capture is not the one of its replays
            return api._empty((need,), torch.uint8, self.k.device, stream)
        handle = api._stream(stream, self.k)
        ws = self._ws.get(handle)
        if ws is None or ws.numel() < need:
            need = need if ws is None else max(need, 2 * ws.numel())
            ws = self._ws[handle] = api._empty((need,), torch.uint8, self.k.device, stream)
        return ws

    def attend(self, q: torch.Tensor, new_off: torch.Tensor, max_new: int, max_len: int,
               mask: Optional[torch.Tensor] = None, scale: Optional[float] = None,
               out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """Attention of the new tokens (already appended) over the cache.  max_len: the most
        cached plus new tokens of a sequence as far as the host knows it (sets how the work is
        split).  scale: head_dim ** -0.5 unless given."""
        if out is None:
            out = api._empty(q.shape, q.dtype, q.device, stream)
        api.moe_tree_attention(self.desc, self.table, self.lens, new_off, max_new, max_len, q, out,
                               q.shape[2] ** -0.5 if scale is None else scale, mask,
                               self._workspace(q.shape[1], max_new, max_len, stream), self.status, stream)
        return out

    def keep(self, new_off: torch.Tensor, keep: torch.Tensor, n_keep: torch.Tensor,
             len_out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """Move the accepted drafts together behind the cached tokens; returns the new
        lengths.  `lens` itself changes only when the caller copies them there, after the
        last layer's cache has been kept."""
        if len_out is None:
            len_out = api._empty(self.lens.shape, self.lens.dtype, self.lens.device, stream)
        api.moe_cache_keep(self.desc, self.table, self.lens, new_off, keep, n_keep, len_out, self.status, stream)
        return len_out


class DecoderBlock:
    """One decoder layer: attention with 4-bit projections over a PagedCache, then the
    mixed-precision expert FFN of a MoELayer, with a norm before and (optionally) after
    each of the two, a gate per channel and a residual scale.

    wqkv fp32 [(n_q_heads + 2 n_kv_heads) head_dim][d_model], wo fp32 [d_model][n_q_heads
    head_dim]; norms: dict of fp32 [d_model] with "attn" and "ffn" (before the blocks) and,
    where the model has them, "attn_post", "ffn_post", "attn_gate", "ffn_gate".
    """

    def __init__(self, moe, wqkv: torch.Tensor, wo: torch.Tensor, n_q_heads: int, n_kv_heads: int, head_dim: int,
                 norms: Dict[str, torch.Tensor], cos: Optional[torch.Tensor] = None,
                 sin: Optional[torch.Tensor] = None, group: int = 128, residual_scale: float = 1.0,
                 branch_scale: float = 1.0, eps: float = 1e-6):
        self.moe, self.norms, self.eps = moe, norms, eps
        self.Hq, self.Hkv, self.D = n_q_heads, n_kv_heads, head_dim
        if wqkv.shape[0] != (n_q_heads + 2 * n_kv_heads) * head_dim or wo.shape[1] != n_q_heads * head_dim:
            raise MoEError("the projections do not fit %d + 2 x %d heads of %d" % (n_q_heads, n_kv_heads, head_dim))
        self.wqkv, self.wo = QuantLinear(wqkv, group), QuantLinear(wo, group)
        self.cos, self.sin = cos, sin
        self.scales = dict(residual_scale=residual_scale, branch_scale=branch_scale)

    def status_value(self) -> int:
        """0, or MOE_ERR_RANGE once the expert layer, whose operands are fp16 for many tokens,
        has met a value beyond fp16's range: that call's outputs are not valid.  Reads it
        back.  (What the cache has met is in its own status_value.)"""
        return self.moe.ffn_status_value()

    def attention(self, h: torch.Tensor, cache: PagedCache, new_off: torch.Tensor, max_new: int, max_len: int,
                  positions: Optional[torch.Tensor] = None, mask: Optional[torch.Tensor] = None,
                  stream=None) -> torch.Tensor:
        """h bf16 [tokens][d_model] (normed) -> the attention block's output, bf16."""
        N, Hq, Hkv, D = h.shape[0], self.Hq, self.Hkv, self.D
        qkv = self.wqkv(h, stream=stream).view(N, Hq + 2 * Hkv, D)
        q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
        q = cache.append(q, k, v, new_off, max_new, positions, self.cos, self.sin, stream=stream)
        o = cache.attend(q, new_off, max_new, max_len, mask, 1.0 / math.sqrt(D), stream=stream)
        return self.wo(o.view(N, Hq * D), stream=stream)

    def forward(self, r: torch.Tensor, h: torch.Tensor, cache: PagedCache, new_off: torch.Tensor, max_new: int,
                max_len: int, positions: Optional[torch.Tensor] = None, mask: Optional[torch.Tensor] = None,
                next_norm: Optional[torch.Tensor] = None, stream=None) -> None:
        """One layer over the new tokens, in place: r [tokens][d_model] is the residual
        stream, h bf16 of the same shape its norm before this layer (moe_block_norm with
        norms["attn"]); afterwards h is the norm before the next one (next_norm).  Calls on
        different streams, and replays of different graphs, are independent, each over a
        cache and tokens of its own."""
        n = self.norms
        a = self.attention(h, cache, new_off, max_new, max_len, positions, mask, stream)
        api.moe_block_norm(r, h, y=a, w_post=n.get("attn_post"), gate=n.get("attn_gate"), w_pre=n["ffn"], r_out=r,
                           eps=self.eps, stream=stream, **self.scales)
        y = self.moe.forward(h, stream=stream, buffers=self.moe.stream_buffers(h.shape[0], stream))
        api.moe_block_norm(r, h, y=y, w_post=n.get("ffn_post"), gate=n.get("ffn_gate"), w_pre=next_norm, r_out=r,
                           eps=self.eps, stream=stream, **self.scales)
