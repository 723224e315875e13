"""The decode step over a tree of drafted tokens: the library's tree operators
on torch tensors.

One step of a model whose cache is ``pool`` [layers, 2, pages, kv_heads, 16,
head_dim] (bf16 or fp16)::

    mask, pos, slots = tree_plan(parents, n_nodes, ctx_len, page_table, n_pages)
    for l in range(layers):
        qkv = ...                                     # [batch * width, (Hq + 2 Hkv) * hd]
        q = qk_norm_rope(qkv, Hq, Hkv, pos.view(-1), slots.view(-1), pool[l, 0], pool[l, 1], inv_freq, ...)
        o = tree_attention(q.view(batch, width, Hq, hd), pool[l, 0], pool[l, 1], page_table, ctx_len, n_nodes, mask)
        ...
    token, logprob = sample(logits, u, temperature, top_k, top_p, min_p)
    accept_len, emitted, ctx_len = tree_commit(token.view(batch, width), tokens, parents, n_nodes, ctx_len,
                                               page_table, pool)

Every call enqueues its work on torch's current stream of the current device
and allocates nothing but its outputs (and the attention's workspace, unless
one is passed) from torch.  Tensors of another stream need torch's own
``record_stream`` or events, as with any torch operation.  Arguments that the
kernels do not support raise ``ValueError`` here or ``PardError`` from the
library; there is no fallback.
"""
from __future__ import annotations

import math
from typing import Optional, Tuple

import torch

from .pard import _check, lib

PAGE = 16
_CODE = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}
_I32, _I64, _F32 = torch.int32, torch.int64, torch.float32


def _stream(t) -> int:
    """The raw current stream; t must lie on the current device."""
    dev = torch._C._cuda_getDevice() if t.is_cuda else -1
    if t.get_device() != dev:
        raise ValueError("tensors must lie on the current CUDA device")
    return torch._C._cuda_getCurrentRawStream(dev)


def _bad(name, t, dtype, shape):
    what = f"{t.dtype} {tuple(t.shape)} on {t.device}" if isinstance(t, torch.Tensor) else type(t).__name__
    raise ValueError(f"{name}: want a contiguous {dtype} tensor of shape {tuple(shape)} on the same device, got {what}")


def _want(name, t, dtype, shape, dev):
    if t.dtype is not dtype or t.shape != shape or t.get_device() != dev or not t.is_contiguous():
        _bad(name, t, dtype, shape)
    return t.data_ptr()


def _cache(name, t, dtype, dev):
    """Pointer and page stride of a [pages, kv_heads, 16, head_dim] cache whose pages may lie apart."""
    if t.dim() != 4 or t.dtype is not dtype or t.get_device() != dev or t.shape[2] != PAGE:
        _bad(name, t, dtype, ("pages", "kv_heads", PAGE, "head_dim"))
    n, h, _, d = t.shape
    s = t.stride()
    if s[3] != 1 or s[2] != d or (h > 1 and s[1] != PAGE * d):
        raise ValueError(f"{name}: each page must be a contiguous [kv_heads, {PAGE}, head_dim] block")
    return t.data_ptr(), s[0] if n > 1 else max(s[0], h * PAGE * d)


def tree_plan(parents, n_nodes, ctx_len, page_table, n_pages: int):
    """Masks, positions and cache slots of tree nodes (pard_tree_plan).

    parents [B, N] int32 (-1: follows the committed tokens), n_nodes [B],
    ctx_len [B], page_table [B, P] int32 over a cache of n_pages pages.
    Returns mask [B, N, ceil(N / 64)] int64, pos [B, N] int32, slots [B, N] int64."""
    st = _stream(parents)
    B, N = parents.shape
    dev = parents.get_device()
    P = page_table.shape[-1]
    mask = torch.empty((B, N, (N + 63) // 64), dtype=_I64, device=parents.device)
    pos = torch.empty((B, N), dtype=_I32, device=parents.device)
    slots = torch.empty((B, N), dtype=_I64, device=parents.device)
    code = lib().pard_tree_plan(
        _want("parents", parents, _I32, (B, N), dev), _want("n_nodes", n_nodes, _I32, (B,), dev),
        _want("ctx_len", ctx_len, _I32, (B,), dev), _want("page_table", page_table, _I32, (B, P), dev), B, N, P,
        n_pages, mask.data_ptr(), pos.data_ptr(), slots.data_ptr(), st)
    if code:
        _check(code, "pard_tree_plan")
    return mask, pos, slots


def rope_frequencies(rot_dim: int, theta: float = 10000.0, scaling: Optional[str] = None, factor: float = 1.0,
                     original_len: int = 8192, low: float = 1.0, high: float = 4.0,
                     device="cuda") -> Tuple[torch.Tensor, float]:
    """inv_freq [rot_dim / 2] (fp32, radians a position) and the amplitude of
    qk_norm_rope, for positions stretched by ``factor`` past ``original_len``:

    ``None``    theta^(-2i/R)
    "linear"    every frequency divided by the factor
    "ntk"       theta raised to theta * factor^(R / (R - 2)): the lowest
                frequency is divided by the factor, the highest kept
    "parts"     frequencies that turn fewer than ``low`` times over
                original_len divided by the factor, more than ``high`` times
                kept, linear in the turns between
    "yarn"      the same with the ramp linear in the pair's index between
                those of ``high`` and ``low`` turns (32 and 1 as a rule), and the
                amplitude 0.1 ln(factor) + 1
    """
    if rot_dim < 2 or rot_dim % 2:
        raise ValueError("rot_dim must be even and positive")
    if not (factor >= 1.0 and theta > 1.0 and original_len > 0):
        raise ValueError("want factor >= 1, theta > 1, original_len > 0")
    i = torch.arange(rot_dim // 2, dtype=torch.float64)
    freq = theta ** (-2.0 * i / rot_dim)
    amplitude = 1.0
    if scaling == "linear":
        freq = freq / factor
    elif scaling == "ntk":
        if rot_dim < 4:
            raise ValueError("ntk scaling needs rot_dim >= 4")
        freq = (theta * factor ** (rot_dim / (rot_dim - 2.0))) ** (-2.0 * i / rot_dim)
    elif scaling in ("parts", "yarn"):
        if not high > low > 0:
            raise ValueError("want high > low > 0")
        if scaling == "parts":
            keep = ((original_len * freq / (2 * math.pi) - low) / (high - low)).clamp(0.0, 1.0)
        else:
            def pair(turns):
                return rot_dim * math.log(original_len / (turns * 2 * math.pi)) / (2 * math.log(theta))
            a, b = max(math.floor(pair(high)), 0), min(math.ceil(pair(low)), rot_dim - 1)
            keep = 1.0 - ((i - a) / max(b - a, 0.001)).clamp(0.0, 1.0)
            amplitude = 0.1 * math.log(factor) + 1.0
        freq = freq * keep + freq / factor * (1.0 - keep)
    elif scaling is not None:
        raise ValueError(f"unknown scaling {scaling!r}")
    return freq.to(_F32).to(device), amplitude


def qk_norm_rope(qkv, n_q_heads: int, n_kv_heads: int, pos, slots, k_cache, v_cache, inv_freq, q_gain=None,
                 k_gain=None, eps: float = 1e-6, interleaved: bool = False, amplitude: float = 1.0):
    """Norm and rotate the query and key heads of QKV rows, write keys and
    values to the paged caches (pard_qk_norm_rope).

    qkv [T, (Hq + 2 Hkv) * hd] bf16 or fp16, rows may lie apart; pos [T] int32;
    slots [T] int64; caches [pages, Hkv, 16, hd]; inv_freq [rot / 2] fp32
    (rot_dim = 2 * its length; None: no rotation); gains [hd] or None.  Returns
    the queries [T, Hq, hd]."""
    st = _stream(qkv)
    dtype, dev = qkv.dtype, qkv.get_device()
    if qkv.dim() != 2 or qkv.stride(1) != 1 or dtype not in _CODE:
        raise ValueError("qkv: want [tokens, (Hq + 2 Hkv) * hd] rows of bf16 or fp16 with contiguous entries")
    T, width = qkv.shape
    kp, stride = _cache("k_cache", k_cache, dtype, dev)
    vp, v_stride = _cache("v_cache", v_cache, dtype, dev)
    n_pages, heads, _, hd = k_cache.shape
    if stride != v_stride or v_cache.shape != k_cache.shape or heads != n_kv_heads or \
            width != (n_q_heads + 2 * n_kv_heads) * hd:
        raise ValueError("qkv and caches disagree on heads, head_dim, pages or page stride")
    half = 0 if inv_freq is None else inv_freq.shape[0]
    q = torch.empty((T, n_q_heads, hd), dtype=dtype, device=qkv.device)
    code = lib().pard_qk_norm_rope(
        qkv.data_ptr(), qkv.stride(0) if T > 1 else max(width, qkv.stride(0)), _CODE[dtype], T, n_q_heads, n_kv_heads,
        hd, None if q_gain is None else _want("q_gain", q_gain, dtype, (hd,), dev),
        None if k_gain is None else _want("k_gain", k_gain, dtype, (hd,), dev), eps,
        _want("pos", pos, _I32, (T,), dev), _want("slots", slots, _I64, (T,), dev),
        None if not half else _want("inv_freq", inv_freq, _F32, (half,), dev), 2 * half, interleaved, amplitude,
        q.data_ptr(), n_q_heads * hd, kp, vp, stride, n_pages, st)
    if code:
        _check(code, "pard_qk_norm_rope")
    return q


def tree_attention_workspace(batch: int, width: int, n_q_heads: int, n_kv_heads: int, head_dim: int, device="cuda"):
    """A workspace for tree_attention calls of these sizes (or smaller), one at a time."""
    n = lib().pard_tree_attention_workspace_bytes(batch, width, n_q_heads, n_kv_heads, head_dim)
    if n == 0:
        raise ValueError("tree_attention does not support these sizes")
    return torch.zeros(n, dtype=torch.uint8, device=device)


_workspaces = {}  # (device, stream): what calls without a workspace of their own use, one after the other


def _workspace(dev: int, st: int, n: int):
    if torch.cuda.is_current_stream_capturing():  # a graph may run beside later calls: its calls have their own
        return torch.zeros(n, dtype=torch.uint8, device=dev)
    ws = _workspaces.get((dev, st))
    if ws is None or ws.numel() < n:
        ws = _workspaces[dev, st] = torch.zeros(n, dtype=torch.uint8, device=dev)
    return ws


def tree_attention(q, k_cache, v_cache, page_table, ctx_len, n_nodes, mask, scale: Optional[float] = None, out=None,
                   workspace=None):
    """Attention of tree nodes over the paged cache and their ancestors
    (pard_tree_attention).

    q [B, N, Hq, hd] bf16 or fp16 (nodes may lie apart, as columns of a QKV
    projection do); caches [pages, Hkv, 16, hd]; page_table [B, P], ctx_len [B],
    n_nodes [B] int32; mask [B, N, ceil(N / 64)] int64 of tree_plan; scale:
    1 / sqrt(hd) unless given; workspace: of tree_attention_workspace (without
    one, calls share one a stream).  Returns [B, N, Hq, hd]."""
    st = _stream(q)
    dtype, dev = q.dtype, q.get_device()
    if q.dim() != 4 or dtype not in _CODE:
        raise ValueError("q: want [batch, width, query heads, head_dim] of bf16 or fp16")
    B, N, Hq, hd = q.shape
    s = q.stride()
    node = s[1] if N > 1 else (s[0] if B > 1 else Hq * hd)
    if s[3] != 1 or (Hq > 1 and s[2] != hd) or (B > 1 and s[0] != N * node):
        raise ValueError("q: a node's heads must be contiguous and nodes evenly spaced")
    kp, stride = _cache("k_cache", k_cache, dtype, dev)
    vp, v_stride = _cache("v_cache", v_cache, dtype, dev)
    n_pages, Hkv, _, d = k_cache.shape
    if stride != v_stride or v_cache.shape != k_cache.shape or d != hd:
        raise ValueError("q and caches disagree on head_dim, pages or page stride")
    P = page_table.shape[-1]
    L = lib()
    if workspace is None:
        workspace = _workspace(dev, st, L.pard_tree_attention_workspace_bytes(B, N, Hq, Hkv, hd))
    if out is None:
        out = torch.empty((B, N, Hq, hd), dtype=dtype, device=q.device)
    code = L.pard_tree_attention(
        q.data_ptr(), node, _CODE[dtype], B, N, Hq, Hkv, hd, kp, vp, stride, n_pages,
        _want("page_table", page_table, _I32, (B, P), dev), P, _want("ctx_len", ctx_len, _I32, (B,), dev),
        _want("n_nodes", n_nodes, _I32, (B,), dev), _want("mask", mask, _I64, (B, N, (N + 63) // 64), dev),
        hd ** -0.5 if scale is None else scale, _want("out", out, dtype, (B, N, Hq, hd), dev), workspace.data_ptr(),
        workspace.numel(), st)
    if code:
        _check(code, "pard_tree_attention")
    return out


def sample(logits, u, temperature=None, top_k=None, top_p=None, min_p=None):
    """One token a row with temperature, top-k, top-p and min-p from given
    uniform numbers (pard_sample).

    logits [R, V] fp32, bf16 or fp16 (rows may lie apart); u [R] fp32 in
    [0, 1); temperature, top_p, min_p [R] fp32, top_k [R] int32, each or None.
    Returns token [R] int32 (-1: a row with no entry above -inf) and its
    log-probability among the entries kept [R] fp32."""
    st = _stream(logits)
    dtype, dev = logits.dtype, logits.get_device()
    if logits.dim() != 2 or logits.stride(1) != 1 or dtype not in _CODE:
        raise ValueError("logits: want [rows, vocab] of fp32, bf16 or fp16 with contiguous rows")
    R, V = logits.shape
    row = (R,)
    token = torch.empty(R, dtype=_I32, device=logits.device)
    logprob = torch.empty(R, dtype=_F32, device=logits.device)
    code = lib().pard_sample(
        logits.data_ptr(), logits.stride(0) if R > 1 else max(V, logits.stride(0)), _CODE[dtype], R, V,
        _want("u", u, _F32, row, dev),
        None if temperature is None else _want("temperature", temperature, _F32, row, dev),
        None if top_k is None else _want("top_k", top_k, _I32, row, dev),
        None if top_p is None else _want("top_p", top_p, _F32, row, dev),
        None if min_p is None else _want("min_p", min_p, _F32, row, dev), token.data_ptr(), logprob.data_ptr(), st)
    if code:
        _check(code, "pard_sample")
    return token, logprob


def tree_commit(sampled, tokens, parents, n_nodes, ctx_len, page_table, pool):
    """Follow the drawn tokens down each tree and compact the path's keys and
    values in the pool, in place (pard_tree_commit).

    sampled, tokens, parents [B, N], n_nodes, ctx_len [B], page_table [B, P]
    int32; pool [layers, 2, pages, Hkv, 16, hd] bf16 or fp16.  Returns
    accept_len [B], emitted [B, N] (-1 after the emitted tokens) and the new
    context lengths [B]."""
    st = _stream(sampled)
    dev = sampled.get_device()
    B, N = sampled.shape
    P = page_table.shape[-1]
    if pool.dim() != 6 or pool.shape[1] != 2 or pool.shape[4] != PAGE or pool.get_device() != dev or \
            pool.dtype not in (torch.bfloat16, torch.float16):
        raise ValueError("pool: want [layers, 2, pages, kv_heads, 16, head_dim] of bf16 or fp16 on the same device")
    L, _, n_pages, Hkv, _, hd = pool.shape
    s = pool.stride()
    if s[5] != 1 or s[4] != hd or (Hkv > 1 and s[3] != PAGE * hd):
        raise ValueError("pool: each page must be a contiguous [kv_heads, 16, head_dim] block")
    accept = torch.empty(B, dtype=_I32, device=sampled.device)
    emitted = torch.empty((B, N), dtype=_I32, device=sampled.device)
    length = torch.empty(B, dtype=_I32, device=sampled.device)
    code = lib().pard_tree_commit(
        _want("sampled", sampled, _I32, (B, N), dev), _want("tokens", tokens, _I32, (B, N), dev),
        _want("parents", parents, _I32, (B, N), dev), _want("n_nodes", n_nodes, _I32, (B,), dev),
        _want("ctx_len", ctx_len, _I32, (B,), dev), _want("page_table", page_table, _I32, (B, P), dev), B, N, P,
        pool.data_ptr(), s[0], s[1], s[2] if n_pages > 1 else Hkv * PAGE * hd, L, Hkv, hd, n_pages,
        accept.data_ptr(), emitted.data_ptr(), length.data_ptr(), st)
    if code:
        _check(code, "pard_tree_commit")
    return accept, emitted, length
