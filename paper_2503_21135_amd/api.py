"""Python names of the C ABI (include/moe_quant.h), taking torch tensors.

torch supplies device memory and the stream only; each function marshals its
arguments into the matching ``extern "C"`` entry point of libmoe_quant.so and
raises MoEError on a non-zero status.  Integer bit patterns (packed codes,
{scale, zero} words) live in int32 tensors; bf16 activations in bfloat16
tensors.
"""
from __future__ import annotations

import ctypes as C
from typing import Optional, Tuple

import numpy as np
import torch

from ._lib import TYPE_BF16, TYPE_FP16, TYPE_FP32, CacheDesc, LayerDesc, MoEError, check, load, stream_capturing


def _p(t: Optional[torch.Tensor]):
    return None if t is None else C.c_void_p(t.data_ptr())


def _s(stream) -> C.c_void_p:
    if stream is None:
        stream = torch.cuda.current_stream()
    return C.c_void_p(stream.cuda_stream)


def _need_cuda(*ts):
    for t in ts:
        if t is not None and not t.is_cuda:
            raise MoEError("expected a device tensor")


def moe_quant_pack(w: torch.Tensor, bits: int, group: int, codes: torch.Tensor,
                   sz: torch.Tensor, n: Optional[int] = None,
                   rows: Optional[torch.Tensor] = None, ld_codes: Optional[int] = None,
                   sz_row_stride: Optional[int] = None, sz_group_stride: int = 1,
                   status: Optional[torch.Tensor] = None, stream=None) -> None:
    """Quantize rows of fp32 w [R][K] at `bits` and pack them (Sec. IV-A, V-B)."""
    _need_cuda(w, codes, sz, rows, status)
    R, K = w.shape
    n = (R if rows is None else rows.numel()) if n is None else n
    ld = K * bits // 32 if ld_codes is None else ld_codes
    srs = K // group if sz_row_stride is None else sz_row_stride
    st = load().moe_quant_pack(_p(w), w.stride(0), R, K, bits, group, _p(rows), n,
                               _p(codes), ld, _p(sz), srs, sz_group_stride, _p(status),
                               _s(stream))
    check(st, "moe_quant_pack")


def moe_code_row_words(K: int, bits: int) -> int:
    """Row stride (32-bit words) of packed code matrices read by the FFN."""
    n = int(load().moe_code_row_words(K, bits))
    if n <= 0:
        raise MoEError("moe_code_row_words: bad K=%d or bits=%d" % (K, bits))
    return n


def moe_route_workspace_bytes(T: int, E: int, k: int, S: int) -> int:
    return int(load().moe_route_workspace_bytes(T, E, k, S))


def moe_route_permute(x: torch.Tensor, w_router: torch.Tensor, bias: Optional[torch.Tensor],
                      k: int, S: int, topk_ids: torch.Tensor, topk_w: torch.Tensor,
                      offsets: torch.Tensor, perm_token: torch.Tensor, inv_perm: torch.Tensor,
                      ws: torch.Tensor, x_perm: Optional[torch.Tensor] = None,
                      stream=None) -> None:
    """Router, top-k and permutation into per-expert segments (Sec. II-A)."""
    _need_cuda(x, w_router, bias, topk_ids, topk_w, offsets, perm_token, inv_perm, ws, x_perm)
    T, d = x.shape
    E = w_router.shape[0]
    st = load().moe_route_permute(_p(x), T, d, _p(w_router), _p(bias), E, k, S, _p(topk_ids),
                                  _p(topk_w), _p(offsets), _p(perm_token), _p(inv_perm),
                                  _p(x_perm), _p(ws), ws.numel() * ws.element_size(), _s(stream))
    check(st, "moe_route_permute")


def moe_ffn_plan(desc: LayerDesc, T: int, k: int) -> Tuple[int, int]:
    ns = C.c_int32(0)
    wb = C.c_size_t(0)
    check(load().moe_ffn_plan(C.byref(desc), T, k, C.byref(ns), C.byref(wb)), "moe_ffn_plan")
    return int(ns.value), int(wb.value)


def moe_expert_ffn_mixed(desc: LayerDesc, x: torch.Tensor, k: int, offsets: torch.Tensor,
                         perm_token: torch.Tensor, o: torch.Tensor, ws: torch.Tensor,
                         status: Optional[torch.Tensor] = None, stream=None) -> None:
    """Grouped mixed-precision SiLU-GLU expert FFN (Sec. IV-A, IV-B, V-B).
    `status` (device int32, optional) receives MOE_ERR_RANGE when the fp16
    operand path meets a value beyond fp16's range."""
    _need_cuda(x, offsets, perm_token, o, ws, status)
    T = x.shape[0]
    st = load().moe_expert_ffn_mixed(C.byref(desc), _p(x), T, k, _p(offsets), _p(perm_token),
                                     _p(o), _p(ws), ws.numel() * ws.element_size(), _p(status),
                                     _s(stream))
    check(st, "moe_expert_ffn_mixed")


def moe_expert_ffn_mixed_ev(desc: LayerDesc, x: torch.Tensor, k: int, offsets: torch.Tensor,
                            perm_token: torch.Tensor, o: torch.Tensor, ws: torch.Tensor,
                            events, status: Optional[torch.Tensor] = None, stream=None) -> None:
    """moe_expert_ffn_mixed recording caller-created hipEvent_t handles
    (a ctypes c_void_p array) at its stage boundaries."""
    _need_cuda(x, offsets, perm_token, o, ws, status)
    T = x.shape[0]
    st = load().moe_expert_ffn_mixed_ev(C.byref(desc), _p(x), T, k, _p(offsets), _p(perm_token),
                                        _p(o), _p(ws), ws.numel() * ws.element_size(), _p(status),
                                        _s(stream), C.cast(events, C.c_void_p), len(events))
    check(st, "moe_expert_ffn_mixed_ev")


def moe_expert_ffn_mixed_noalloc(desc: LayerDesc, x: torch.Tensor, k: int, offsets: torch.Tensor,
                                 perm_token: torch.Tensor, o: torch.Tensor,
                                 status: Optional[torch.Tensor] = None, stream=None) -> None:
    """moe_expert_ffn_mixed with the library's fixed per-GPU workspace
    (no workspace argument, no allocation)."""
    _need_cuda(x, offsets, perm_token, o, status)
    T = x.shape[0]
    st = load().moe_expert_ffn_mixed_noalloc(C.byref(desc), _p(x), T, k, _p(offsets),
                                             _p(perm_token), _p(o), _p(status), _s(stream))
    check(st, "moe_expert_ffn_mixed_noalloc")


def moe_set_channel_switch(desc: LayerDesc, kind: int, slots_on: Optional[np.ndarray],
                           stream=None) -> None:
    """Install cached copies by (expert, row) header (Sec. IV-B, V-A)."""
    if slots_on is None or len(slots_on) == 0:
        arr, ptr, n = None, None, 0
    else:
        arr = np.ascontiguousarray(slots_on, dtype=np.int32)
        ptr, n = arr.ctypes.data_as(C.c_void_p), int(arr.size)
    st = load().moe_set_channel_switch(C.byref(desc), kind, ptr, n, _s(stream))
    check(st, "moe_set_channel_switch")


def moe_requant_channels(desc: LayerDesc, kind: int, cache: torch.Tensor,
                         expert_bits: np.ndarray, status: Optional[torch.Tensor] = None,
                         stream=None) -> None:
    """Requantize the cached 16-bit channels of one kind into its copy slots at
    each expert's new precision (Sec. IV-B, requantization for new datasets).

    cache        device float16 [n_slots][K] (row s = original channel of slot s)
    expert_bits  int [n_experts], 0 = leave that expert's slots as they are
    """
    _need_cuda(cache, status)
    if cache.dtype != torch.float16 or cache.dim() != 2 or cache.stride(1) != 1:
        raise MoEError("cache must be a row-major float16 matrix")
    eb = np.ascontiguousarray(expert_bits, dtype=np.int32)
    if eb.size != desc.n_experts:
        raise MoEError("expert_bits needs one entry per routed expert")
    st = load().moe_requant_channels(C.byref(desc), kind, _p(cache), cache.stride(0),
                                     eb.ctypes.data_as(C.c_void_p), _p(status), _s(stream))
    check(st, "moe_requant_channels")


def moe_unpermute_combine(o: torch.Tensor, n_split: int, inv_perm: torch.Tensor,
                          topk_w: torch.Tensor, k: int, S: int, y: torch.Tensor,
                          stream=None) -> None:
    """y[t] = sum_j w[t][j] o[inv[t][j]] + sum_s o[inv[t][k+s]]."""
    _need_cuda(o, inv_perm, topk_w, y)
    T, d = y.shape
    split_stride = o.stride(0) if o.dim() == 3 else o.numel()
    st = load().moe_unpermute_combine(_p(o), n_split, split_stride, _p(inv_perm), _p(topk_w),
                                      T, k, S, d, _p(y), _s(stream))
    check(st, "moe_unpermute_combine")


# ---------------------------------------------------------------------------
# decoder block around the expert FFN
# ---------------------------------------------------------------------------
# These calls take a few microseconds on the device, so their marshalling passes
# plain integers (ctypes takes them for pointers) and checks only what the C entry
# points cannot see: types, shapes and strides of the tensors.
_TYPES = {torch.bfloat16: TYPE_BF16, torch.float16: TYPE_FP16, torch.float32: TYPE_FP32}


def _type(t: torch.Tensor, what: str) -> int:
    ty = _TYPES.get(t.dtype)
    if ty is None:
        raise MoEError("%s must be bfloat16, float16 or float32, not %s" % (what, t.dtype))
    return ty


def _stream(stream, t: torch.Tensor) -> int:
    """Handle of the stream to work on: the current one of t's device unless given (asked
    for as a number: the Stream object of torch.cuda.current_stream costs 3 us)."""
    return torch._C._cuda_getCurrentRawStream(t.get_device()) if stream is None else stream.cuda_stream


def _capturing(stream) -> bool:
    """Whether what is launched on the stream (None: the current one) goes into a graph."""
    return torch.cuda.is_current_stream_capturing() if stream is None else stream_capturing(stream.cuda_stream)


def _empty(shape, dtype: torch.dtype, device, stream) -> torch.Tensor:
    """A new tensor whose memory is reused in the order of the stream that works on it."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _rows(t: torch.Tensor, T: int, n: int, what: str) -> Tuple[int, int]:
    """(data pointer, row stride) of a [T][n] device tensor whose rows are contiguous."""
    if t.shape == (T, n) and t.is_cuda:
        s = t.stride()
        if s[1] == 1 or n <= 1:
            return t.data_ptr(), s[0] if T > 1 else n
    raise MoEError("%s must be a device tensor of shape (%d, %d) with contiguous rows" % (what, T, n))


def _flat(t: Optional[torch.Tensor], shape: tuple, dtype: torch.dtype, what: str):
    """Data pointer of a contiguous device tensor (None for None)."""
    if t is None:
        return None
    if t.dtype is dtype and t.shape == shape and t.is_cuda and t.is_contiguous():
        return t.data_ptr()
    raise MoEError("%s must be a contiguous %s device tensor of shape %s" % (what, dtype, tuple(shape)))


def moe_quant_linear(x: torch.Tensor, codes: torch.Tensor, sz: torch.Tensor, y: torch.Tensor,
                     bits: int = 4, bias: Optional[torch.Tensor] = None, stream=None) -> None:
    """y [T][R] = x [T][K] times packed 4-bit rows (+ bias [R]).

    codes  int32 [R][>= K/8], a row's words contiguous (moe_quant_pack's layout)
    sz     int32 [K/group][R] {scale, zero} words; a transposed view of [R][K/group] works too
    x      bfloat16 or float16; y the same type or float32
    """
    T, K = x.shape
    G, R = sz.shape
    if G < 1 or K % G:
        raise MoEError("sz has %d groups for K = %d" % (G, K))
    if codes.dtype is not torch.int32 or sz.dtype is not torch.int32 or not sz.is_cuda:
        raise MoEError("codes and sz must be int32 device tensors")
    words = codes.shape[-1]
    if words * 8 < K:
        raise MoEError("codes have shape %s for %d rows of K = %d" % (tuple(codes.shape), R, K))
    sg, sr = sz.stride()
    xp, ld_x = _rows(x, T, K, "x")
    cp, ld_c = _rows(codes, R, words, "codes")
    yp, ld_y = _rows(y, T, R, "y")
    st = load().moe_quant_linear(xp, _type(x, "x"), ld_x, T, K, cp, ld_c if R > 1 else K // 8,
                                 sz.data_ptr(), sr if R > 1 else 1, sg if G > 1 else R, R, bits, K // G,
                                 _flat(bias, (R,), torch.float32, "bias"), yp, _type(y, "y"), ld_y, _stream(stream, x))
    if st:
        check(st, "moe_quant_linear")


def moe_block_norm(r: torch.Tensor, h: Optional[torch.Tensor] = None, y: Optional[torch.Tensor] = None,
                   w_post: Optional[torch.Tensor] = None, gate: Optional[torch.Tensor] = None,
                   w_pre: Optional[torch.Tensor] = None, r_out: Optional[torch.Tensor] = None,
                   branch_scale: float = 1.0, residual_scale: float = 1.0, eps: float = 1e-6,
                   stream=None) -> None:
    """Norm after a block, gate, residual add and norm before the next, for rows [T][d]:
    v = residual_scale r + branch_scale gate rms(y) w_post;  r_out = v;  h = rms(v) w_pre.

    gate is [d] (per channel), [T][1] (per token) or [T][d]; without y, v is the scaled
    residual alone; without w_post, y is taken as it is.  r_out and h may each be r, y or a
    gate per element, in place.
    """
    T, d = r.shape
    g, g_type, g_row, g_col = None, 0, 0, 0
    if gate is not None:
        g_type = _type(gate, "gate")
        if gate.dim() == 1:
            g, g_col = _rows(gate[None], 1, d, "gate")[0], 1
        elif gate.shape[1] == 1 and d > 1:
            g, g_row = _rows(gate, T, 1, "gate")
        else:
            (g, g_row), g_col = _rows(gate, T, d, "gate"), 1
    yp, ld_y, y_type = None, d, 0
    if y is not None:
        (yp, ld_y), y_type = _rows(y, T, d, "y"), _type(y, "y")
    op, ld_o = None, d
    if r_out is not None:
        if r_out.dtype is not r.dtype:
            raise MoEError("r_out must have the type of r")
        op, ld_o = _rows(r_out, T, d, "r_out")
    hp, ld_h, h_type = None, d, 0
    if h is not None:
        (hp, ld_h), h_type = _rows(h, T, d, "h"), _type(h, "h")
    rp, ld_r = _rows(r, T, d, "r")
    st = load().moe_block_norm(yp, y_type, ld_y, rp, _type(r, "r"), ld_r, T, d,
                               _flat(w_post, (d,), torch.float32, "w_post"), g, g_type, g_row, g_col, branch_scale,
                               residual_scale, _flat(w_pre, (d,), torch.float32, "w_pre"), eps, op, ld_o, hp, h_type,
                               ld_h, _stream(stream, r))
    if st:
        check(st, "moe_block_norm")


def _heads(t: torch.Tensor, N: int, H: int, D: int, dtype: torch.dtype, what: str) -> Tuple[int, int]:
    """(data pointer, token stride) of a [N][H][D] device tensor whose heads lie side by side."""
    if t.dtype is dtype and t.shape == (N, H, D) and t.is_cuda:
        s = t.stride()
        if s[2] == 1 and (s[1] == D or H <= 1):
            return t.data_ptr(), s[0] if N > 1 else H * D
    raise MoEError("%s must be a %s device tensor of shape (%d, %d, %d), the heads of a token side by side"
                   % (what, dtype, N, H, D))


def _batch(table: torch.Tensor, lens: torch.Tensor, new_off: torch.Tensor):
    """(table, max_pages, cache_len, n_seqs, new_off) of the three cache calls."""
    B = lens.shape[0]
    if table.dim() != 2:
        raise MoEError("table must be [sequences][pages]")
    return (_flat(table, (B, table.shape[1]), torch.int32, "table"), table.shape[1],
            _flat(lens, (B,), torch.int32, "cache_len"), B, _flat(new_off, (B + 1,), torch.int32, "new_off"))


_DTYPE16 = {TYPE_BF16: torch.bfloat16, TYPE_FP16: torch.float16}


def moe_cache_append(desc: CacheDesc, table: torch.Tensor, lens: torch.Tensor, new_off: torch.Tensor,
                     max_new: int, q: Optional[torch.Tensor], k: torch.Tensor, v: torch.Tensor,
                     q_out: Optional[torch.Tensor], positions: Optional[torch.Tensor] = None,
                     cos: Optional[torch.Tensor] = None, sin: Optional[torch.Tensor] = None,
                     interleaved: bool = False, status: Optional[torch.Tensor] = None, stream=None) -> None:
    """Rotate q and k [tokens][heads][head_dim] by cos/sin [max_pos][rot_dim/2] and store
    k and v of the new tokens in the cache."""
    N, dt, D, Hkv = k.shape[0], _DTYPE16[desc.type], desc.head_dim, desc.n_heads
    if (q is None) != (q_out is None) or (cos is None) != (sin is None):
        raise MoEError("q and q_out, cos and sin come in pairs")
    tab = (1, 0) if cos is None else tuple(cos.shape)
    qp, ld_q, Hq, op, ld_o = None, 0, 0, None, 0
    if q is not None:
        Hq = q.shape[1]
        qp, ld_q = _heads(q, N, Hq, D, dt, "q")
        op, ld_o = _heads(q_out, N, Hq, D, dt, "q_out")
    kp, ld_k = _heads(k, N, Hkv, D, dt, "k")
    vp, ld_v = _heads(v, N, Hkv, D, dt, "v")
    st = load().moe_cache_append(
        C.byref(desc), *_batch(table, lens, new_off), N, max_new, qp, ld_q, Hq, kp, ld_k, vp, ld_v,
        _flat(positions, (N,), torch.int32, "positions"), _flat(cos, tab, torch.float32, "cos"),
        _flat(sin, tab, torch.float32, "sin"), 2 * tab[1], tab[0], int(interleaved), op, ld_o,
        _flat(status, (1,), torch.int32, "status"), _stream(stream, k))
    if st:
        check(st, "moe_cache_append")


def moe_tree_attention_plan(desc: CacheDesc, n_q_heads: int, n_seqs: int, max_new: int,
                            max_len: int) -> Tuple[int, int]:
    """(parts the keys are split into, workspace bytes) of moe_tree_attention."""
    ns, wb = C.c_int32(0), C.c_size_t(0)
    check(load().moe_tree_attention_plan(C.byref(desc), n_q_heads, n_seqs, max_new, max_len, C.byref(ns),
                                         C.byref(wb)), "moe_tree_attention_plan")
    return int(ns.value), int(wb.value)


def moe_tree_attention(desc: CacheDesc, table: torch.Tensor, lens: torch.Tensor, new_off: torch.Tensor,
                       max_new: int, max_len: int, q: torch.Tensor, out: torch.Tensor, scale: float,
                       mask: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None,
                       status: Optional[torch.Tensor] = None, stream=None) -> None:
    """Attention of the new tokens q [tokens][heads][head_dim] over the cache.  mask is
    int64 [tokens][words]: bit m of a token's words, m % 64 of word m // 64, lets it see
    its sequence's new token m; None is a chain (each token sees itself and those before)."""
    N, Hq, D = q.shape
    if D != desc.head_dim:
        raise MoEError("q has heads of %d, the cache of %d" % (D, desc.head_dim))
    dt = _DTYPE16[desc.type]
    words = 0 if mask is None else mask.shape[-1]
    qp, ld_q = _heads(q, N, Hq, D, dt, "q")
    op, ld_o = _heads(out, N, Hq, D, dt, "out")
    wp, wb = None, 0
    if ws is not None:
        if not ws.is_cuda or not ws.is_contiguous():
            raise MoEError("ws must be a contiguous device tensor")
        wp, wb = ws.data_ptr(), ws.numel() * ws.element_size()
    st = load().moe_tree_attention(
        C.byref(desc), *_batch(table, lens, new_off), N, max_new, max_len, qp, ld_q, Hq,
        _flat(mask, (N, words), torch.int64, "mask"), words, scale, op, ld_o,
        _flat(status, (1,), torch.int32, "status"), wp, wb, _stream(stream, q))
    if st:
        check(st, "moe_tree_attention")


def moe_cache_keep(desc: CacheDesc, table: torch.Tensor, lens: torch.Tensor, new_off: torch.Tensor,
                   keep: torch.Tensor, n_keep: torch.Tensor, len_out: Optional[torch.Tensor] = None,
                   status: Optional[torch.Tensor] = None, stream=None) -> None:
    """Move the accepted drafts keep [sequences][max_keep] (the first n_keep of each row,
    ascending) together behind the cached tokens."""
    B = lens.shape[0]
    st = load().moe_cache_keep(
        C.byref(desc), *_batch(table, lens, new_off), _flat(keep, (B, keep.shape[-1]), torch.int32, "keep"),
        keep.shape[-1], _flat(n_keep, (B,), torch.int32, "n_keep"), _flat(len_out, (B,), torch.int32, "len_out"),
        _flat(status, (1,), torch.int32, "status"), _stream(stream, lens))
    if st:
        check(st, "moe_cache_keep")


# ---------------------------------------------------------------------------
# offline bit allocation (host only)
# ---------------------------------------------------------------------------
def _np_ptr(a: np.ndarray) -> C.c_void_p:
    return a.ctypes.data_as(C.c_void_p)


def moe_expert_significance(sig: np.ndarray, topk_ids: np.ndarray, n_experts: int):
    """Eq. (1): (s_exp float64 [E], token share float64 [E]) of one dataset."""
    sig = np.ascontiguousarray(sig, np.float32)
    ids = np.ascontiguousarray(topk_ids, np.int32)
    if ids.ndim != 2 or ids.shape[0] != sig.shape[0]:
        raise MoEError("topk_ids must be [T][k] with T = len(sig)")
    s = np.empty(n_experts, np.float64)
    sh = np.empty(n_experts, np.float64)
    st = load().moe_expert_significance(_np_ptr(sig), _np_ptr(ids), ids.shape[0], ids.shape[1],
                                        n_experts, _np_ptr(s), _np_ptr(sh))
    check(st, "moe_expert_significance")
    return s, sh


def moe_allocate_bits(x: np.ndarray, share: np.ndarray, levels=(8, 4, 3, 2), m: float = 2.0,
                      eps: float = 1e-9, max_iter: int = 300, alpha: float = 0.3) -> dict:
    """Alg. 1 + cluster precision + low-precision-first -> per-expert bits."""
    x = np.ascontiguousarray(x, np.float64)
    share = np.ascontiguousarray(share, np.float64)
    lv = np.ascontiguousarray(levels, np.int32)
    n, c = x.shape[0], lv.shape[0]
    bits = np.empty(n, np.int32)
    V = np.empty(c, np.float64)
    U = np.empty((n, c), np.float64)
    rounds = C.c_int32(0)
    st = load().moe_allocate_bits(_np_ptr(x), _np_ptr(share), n, _np_ptr(lv), c, m, eps,
                                  max_iter, alpha, _np_ptr(bits), _np_ptr(V), _np_ptr(U),
                                  C.byref(rounds))
    check(st, "moe_allocate_bits")
    return dict(bits=bits, V=V, U=U, rounds=int(rounds.value))
