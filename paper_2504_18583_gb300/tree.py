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

Beside the tree, what a serving loop needs around that step: ``chunk_attention``
reads prompts in pieces (or decodes token by token) over the same cache, with a
sliding window and first tokens that stay visible; ``quantized_cache`` is an 8-bit
form of it that ``qk_norm_rope`` writes and ``chunk_attention`` reads; and
``adjust_logits`` applies penalties, biases and grammar masks before ``sample``.

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

from . import pard

pard.lib()  # raises if the library has not been built
try:
    from . import _tree_ops as _ops
except ImportError as e:
    raise RuntimeError("the torch binding of the tree operators is missing: build it with __graft_entry__.build() "
                       "(there is no fallback)") from e
_ops.set_error(pard.PardError)


def tree_plan(parents, n_nodes, ctx_len, page_table, n_pages: int):
    """Masks, positions and cache slots of tree nodes (pard_tree_plan).

    parents [B, N] int32 (-1: follows the committed tokens), n_nodes [B],
    ctx_len [B], page_table [B, P] int32 over a cache of n_pages pages.
    Returns mask [B, N, ceil(N / 64)] int64, pos [B, N] int32, slots [B, N] int64."""
    return _ops.tree_plan(parents, n_nodes, ctx_len, page_table, n_pages)


def rope_frequencies(rot_dim: int, theta: float = 10000.0, scaling: Optional[str] = None, factor: float = 1.0,
                     original_len: int = 8192, low: float = 1.0, high: Optional[float] = None,
                     device="cuda") -> Tuple[torch.Tensor, float]:
    """inv_freq [rot_dim / 2] (fp32, radians a position) and the amplitude of
    qk_norm_rope, for positions stretched by ``factor`` past ``original_len``:

    ``None``    theta^(-2i/R)
    "linear"    every frequency divided by the factor
    "ntk"       theta raised to theta * factor^(R / (R - 2)): the lowest
                frequency is divided by the factor, the highest kept
    "parts"     frequencies that turn fewer than ``low`` times over
                original_len divided by the factor, more than ``high`` times
                (4 unless given) kept, linear in the turns between
    "yarn"      the same with the ramp linear in the pair's index between
                those of ``high`` (32 unless given) and ``low`` turns, and the
                amplitude 0.1 ln(factor) + 1
    """
    if high is None:
        high = 32.0 if scaling == "yarn" else 4.0
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
    return freq.to(torch.float32).to(device), amplitude


def qk_norm_rope(qkv, n_q_heads: int, n_kv_heads: int, pos, slots, k_cache, v_cache, inv_freq, q_gain=None,
                 k_gain=None, eps: float = 1e-6, interleaved: bool = False, amplitude: float = 1.0, k_scale=None,
                 v_scale=None):
    """Norm and rotate the query and key heads of QKV rows, write keys and
    values to the paged caches (pard_qk_norm_rope).

    qkv [T, (Hq + 2 Hkv) * hd] bf16 or fp16, rows may lie apart; pos [T] int32;
    slots [T] int64; caches [pages, Hkv, 16, hd]; inv_freq [rot / 2] fp32
    (rot_dim = 2 * its length; None: no rotation); gains [hd] or None.  With
    k_scale and v_scale [pages, Hkv, 16] (float8_e8m0fnu or uint8) the caches are
    float8_e4m3fn and a token's head is stored as codes and a power of two
    (pard_qk_norm_rope_quantized; quantized_cache makes one); tokens of a call
    then need slots of their own.  chunk_attention reads such entries as fp16: held
    to 65504 and to multiples of 2^-24.  Returns the queries [T, Hq, hd]."""
    return _ops.qk_norm_rope(qkv, n_q_heads, n_kv_heads, pos, slots, k_cache, v_cache, inv_freq, q_gain, k_gain, eps,
                             interleaved, amplitude, k_scale, v_scale)


def quantized_cache(n_pages: int, n_kv_heads: int, head_dim: int, device="cuda"):
    """One layer's 8-bit cache: k_cache, v_cache [pages, Hkv, 16, hd] float8_e4m3fn, zeros, and k_scale, v_scale [pages, Hkv, 16]
    float8_e8m0fnu, ones (a token's head takes hd + 1 bytes of each; the entry is its code times its scale)."""
    def bytes_of(value, *shape):
        return torch.full(shape, value, dtype=torch.uint8, device=device)
    shape = (n_pages, n_kv_heads, 16)
    k, v = (bytes_of(0, *shape, head_dim).view(torch.float8_e4m3fn) for _ in range(2))
    k_scale, v_scale = (bytes_of(127, *shape).view(torch.float8_e8m0fnu) for _ in range(2))
    return k, v, k_scale, v_scale


def tree_attention_workspace(batch: int, width: int, n_q_heads: int, n_kv_heads: int, head_dim: int, device="cuda"):
    """A workspace for tree_attention calls of these sizes (or smaller), one at a time."""
    n = pard.lib().pard_tree_attention_workspace_bytes(batch, width, n_q_heads, n_kv_heads, head_dim)
    if n == 0:
        raise ValueError("tree_attention does not support these sizes")
    return torch.zeros(n, dtype=torch.uint8, device=device)


def shared_workspace():
    """The workspace that tree_attention and chunk_attention calls without one use on the current stream; None before
    the first.

    Should a wait inside the kernel ever run out (2 s), that call's output is NaN, and so is that of every later call
    with the same workspace.  Once the cause is gone, ``shared_workspace().zero_()`` makes it fit for use again (a
    call that a CUDA graph captured has a workspace of its own, which each replay zeroes)."""
    return _ops.shared_workspace()


def tree_attention(q, k_cache, v_cache, page_table, ctx_len, n_nodes, mask, scale: Optional[float] = None, out=None,
                   workspace=None):
    """Attention of tree nodes over the paged cache and their ancestors
    (pard_tree_attention).

    q [B, N, Hq, hd] bf16 or fp16 (nodes may lie apart, as columns of a QKV
    projection do); caches [pages, Hkv, 16, hd]; page_table [B, P], ctx_len [B],
    n_nodes [B] int32; mask [B, N, ceil(N / 64)] int64 of tree_plan; scale:
    1 / sqrt(hd) unless given; workspace: of tree_attention_workspace (without
    one, calls share one a stream: shared_workspace; a call that a CUDA graph
    captures gets its own, which each replay zeroes, 11 to 43 MB: one that is
    given saves that).  Returns [B, N, Hq, hd]."""
    return _ops.tree_attention(q, k_cache, v_cache, page_table, ctx_len, n_nodes, mask, scale, out, workspace,
                               workspace is None and torch.cuda.is_current_stream_capturing())


def chunk_attention_workspace(n_tokens: int, batch: int, n_q_heads: int, n_kv_heads: int, head_dim: int, device="cuda"):
    """A workspace for chunk_attention calls with these heads and no more tokens and sequences, one at a time."""
    n = pard.lib().pard_chunk_attention_workspace_bytes(n_tokens, batch, n_q_heads, n_kv_heads, head_dim)
    if n == 0:
        raise ValueError("chunk_attention does not support these sizes")
    return torch.zeros(n, dtype=torch.uint8, device=device)


def chunk_attention(q, k_cache, v_cache, page_table, starts, ctx_len, scale: Optional[float] = None, window: int = 0,
                    sinks: int = 0, k_scale=None, v_scale=None, out=None, workspace=None):
    """Attention of a batch's new tokens over their sequences' paged caches
    (pard_chunk_attention): pieces of prompts, single tokens, or both.

    q [T, Hq, hd] bf16 or fp16 (tokens may lie apart), rows starts[b] to
    starts[b + 1] - 1 sequence b's, at positions ctx_len[b], ctx_len[b] + 1, ...,
    their own keys and values in the cache already (qk_norm_rope); caches [pages,
    Hkv, 16, hd] of q's type, or float8_e4m3fn with k_scale and v_scale [pages,
    Hkv, 16]; page_table [B, P], starts [B + 1], ctx_len [B] int32.  A token at
    position p sees the keys j <= p; with window > 0 only those with
    p - j < window or j < sinks.  scale: 1 / sqrt(hd) unless given; workspace: of
    chunk_attention_workspace (without one, calls share the stream's with
    tree_attention: shared_workspace; a call that a CUDA graph captures gets its
    own); out must not lie over q.  Returns [T, Hq, hd]; rows of no sequence are not
    written."""
    return _ops.chunk_attention(q, k_cache, v_cache, page_table, starts, ctx_len, scale, window, sinks, k_scale, v_scale,
                                out, workspace)


def adjust_logits(logits, history=None, hist_len=None, prompt_len=None, repetition=None, frequency=None, presence=None,
                  bias_ids=None, bias=None, allowed=None, tokens=None, mask=None, out=None):
    """What requests ask of their logits before a token is drawn
    (pard_adjust_logits): penalties, biases and a grammar's mask.

    logits [B * N, V] fp32, bf16 or fp16 (rows may lie apart), N rows a sequence:
    its next token's, or its tree's nodes'.  For each sequence: history [B, L]
    int32, of which the first hist_len [B] count and the first prompt_len [B] of
    those are the prompt; repetition, frequency, presence [B] fp32; bias_ids
    [B, M] int32 and bias [B, M] fp32.  For each row: allowed [B * N, ceil(V / 32)]
    int32, a clear bit forbids the token; tokens [B, N] int32 and mask of
    tree_plan: a node's branch counts as generated.  Each may be None.

        z / r if z > 0 else z r   for tokens of the history
        - frequency * count - presence * (count > 0)   of what was generated
        + biases, then -inf where not allowed

    Returns [B * N, V] of the logits' type, or writes `out`, which may be logits (but not lie over others of its entries)."""
    return _ops.adjust_logits(logits, history, hist_len, prompt_len, repetition, frequency, presence, bias_ids, bias,
                              allowed, tokens, mask, out)


def sample(logits, u, temperature=None, top_k=None, top_p=None, min_p=None):
    """One token a row with temperature, top-k, top-p and min-p from given
    uniform numbers (pard_sample).

    logits [R, V] fp32, bf16 or fp16 (rows may lie apart); u [R] fp32 in
    [0, 1); temperature, top_p, min_p [R] fp32, top_k [R] int32, each or None.
    Returns token [R] int32 (-1: a row with no entry above -inf) and its
    log-probability among the entries kept [R] fp32."""
    return _ops.sample(logits, u, temperature, top_k, top_p, min_p)


def tree_commit(sampled, tokens, parents, n_nodes, ctx_len, page_table, pool):
    """Follow the drawn tokens down each tree and compact the path's keys and
    values in the pool, in place (pard_tree_commit).

    sampled, tokens, parents [B, N], n_nodes, ctx_len [B], page_table [B, P]
    int32; pool [layers, 2, pages, Hkv, 16, hd] bf16 or fp16.  Returns
    accept_len [B], emitted [B, N] (-1 after the emitted tokens) and the new
    context lengths [B]."""
    return _ops.tree_commit(sampled, tokens, parents, n_nodes, ctx_len, page_table, pool)
