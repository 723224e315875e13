"""The serving operators' host side: every refusal comes before any CUDA call, so
these run without a GPU, with pointers that are never followed."""
import ctypes
import os
import re

import pytest

from conftest import ROOT

P = 0x10000  # 16-byte aligned, not null
FAR = 1 << 46  # behind anything that starts at P
ARG, SHAPE = -1, -2


@pytest.fixture(scope="module")
def lib():
    from paper_2504_18583_gb300 import _build, pard
    _build.build()
    return pard.lib()


def call(lib, name, good, **edit):
    args = dict(good)
    args.update(edit)
    return getattr(lib, name)(*args.values())


WRITE = dict(qkv=P, qkv_stride=12 * 64, dtype=0, n_tokens=3, hq=8, hkv=2, hd=64, qg=P, kg=None, eps=1e-6, pos=P, slots=P, freq=P,
             rot=64, inter=0, amp=1.0, q=P, q_stride=512, k=P, v=P, page_stride=2 * 16 * 64, ks=P, vs=P, scale_stride=32, n_pages=3,
             stream=None)
CHUNK = dict(q=P, q_stride=512, dtype=0, n_tokens=9, batch=2, hq=8, hkv=2, hd=64, k=P, v=P, page_stride=2048, ks=None, vs=None,
             scale_stride=0, n_pages=3, table=P, max_pages=4, starts=P, ctx=P, window=0, sinks=0, scale=0.125, out=FAR, ws=P,
             ws_bytes=1 << 30, stream=None)
EIGHT = dict(ks=P, vs=P, scale_stride=32)
ADJUST = dict(z=P, stride=100, dtype=2, batch=2, width=3, vocab=100, hist=P, max_hist=10, hist_len=P, prompt=P, rep=P, freq=P, pres=P,
              ids=P, bias=P, n_bias=4, allowed=P, tokens=P, mask=P, out=P, out_stride=100, stream=None)


@pytest.mark.parametrize("name,good,edits", [
    ("pard_qk_norm_rope_quantized", WRITE, [
        (dict(qkv=None), ARG), (dict(freq=None), ARG), (dict(k=None), ARG), (dict(ks=None), ARG), (dict(vs=None), ARG),
        (dict(dtype=2), SHAPE), (dict(hd=96), SHAPE), (dict(rot=72), SHAPE), (dict(rot=128), SHAPE), (dict(scale_stride=16), ARG),
        (dict(scale_stride=40), ARG), (dict(ks=P + 8), ARG), (dict(page_stride=2048 + 8), ARG), (dict(page_stride=1024), SHAPE),
        (dict(qkv_stride=12 * 64 - 8), ARG), (dict(q_stride=500), ARG), (dict(v=P + 8), ARG), (dict(eps=float("nan")), ARG),
        (dict(n_tokens=-1), ARG), (dict(hkv=0), SHAPE), (dict(n_pages=0), SHAPE), (dict(hq=0), SHAPE)]),
    ("pard_chunk_attention", CHUNK, [
        (dict(q=None), ARG), (dict(starts=None), ARG), (dict(ctx=None), ARG), (dict(table=None), ARG), (dict(out=None), ARG),
        (dict(ws=None), ARG), (dict(dtype=2), SHAPE), (dict(hq=7), SHAPE), (dict(hq=8192), SHAPE), (dict(hd=32), SHAPE),
        (dict(batch=0), SHAPE), (dict(batch=65536), SHAPE), (dict(n_tokens=-1), SHAPE), (dict(n_tokens=1 << 29), SHAPE),
        (dict(max_pages=0), ARG), (dict(max_pages=(1 << 26) + 1), ARG), (dict(window=-1), ARG), (dict(sinks=-1), ARG),
        (dict(scale=float("inf")), ARG), (dict(q_stride=504), ARG), (dict(q_stride=514), ARG), (dict(q=P + 4), ARG),
        (dict(out=P + 2), ARG), (dict(ws_bytes=4096), ARG), (dict(page_stride=2052), SHAPE), (dict(page_stride=2000), SHAPE),
        (dict(n_tokens=1 << 27, max_pages=1 << 26), SHAPE), (dict(ks=P), ARG), (dict(vs=P), ARG), (dict(EIGHT, scale_stride=16), ARG),
        (dict(EIGHT, vs=P + 4), ARG), (dict(EIGHT, page_stride=2056), ARG), (dict(n_pages=0), SHAPE),
        # the output over the queries: the same rows, the last row's last entries, a row between rows that lie apart
        (dict(out=P), ARG), (dict(out=P + 2 * 9 * 512 - 16), ARG), (dict(q_stride=512 * 100, out=P + 2 * 512 * 500 - 16), ARG),
        (dict(q=FAR + 2 * 9 * 512 - 16), ARG)]),
    ("pard_adjust_logits", ADJUST, [
        (dict(z=None), ARG), (dict(out=None), ARG), (dict(dtype=3), SHAPE), (dict(batch=-1), ARG), (dict(batch=65536), ARG),
        (dict(batch=65535, width=257), ARG), (dict(vocab=0), SHAPE), (dict(vocab=262145, stride=262145, out_stride=262145), SHAPE),
        (dict(hist=None), ARG), (dict(hist_len=None), ARG), (dict(max_hist=524001), ARG), (dict(max_hist=-1), ARG), (dict(ids=None), ARG),
        (dict(bias=None), ARG), (dict(n_bias=2048), ARG), (dict(n_bias=-1), ARG), (dict(tokens=None), ARG), (dict(mask=None), ARG),
        (dict(width=257), ARG), (dict(stride=99), ARG), (dict(out_stride=99), ARG), (dict(z=P + 2), ARG), (dict(out=P + 1), ARG)]),
])
def test_refusals_without_a_gpu(lib, name, good, edits):
    for edit, code in edits:
        assert call(lib, name, good, **edit) == code, (name, edit)
        assert lib.pard_last_error()


def test_empty_calls_do_nothing(lib):
    assert call(lib, "pard_qk_norm_rope_quantized", WRITE, n_tokens=0, qkv=None) == 0
    assert call(lib, "pard_chunk_attention", CHUNK, n_tokens=0, q=None) == 0
    assert call(lib, "pard_adjust_logits", ADJUST, batch=0, z=None) == 0
    assert call(lib, "pard_adjust_logits", ADJUST, width=0, z=None) == 0


def test_workspace_sizes(lib):
    f, tree = lib.pard_chunk_attention_workspace_bytes, lib.pard_tree_attention_workspace_bytes
    assert f(1, 1, 32, 8, 128) > 4096
    assert f(8191, 1, 32, 8, 128) > f(32, 32, 32, 8, 128)  # two blocks of query vectors
    assert f(32, 32, 32, 8, 64) == tree(50, 32, 32, 8, 64) and f(8191, 1, 64, 8, 128) == tree(1, 256, 64, 8, 128)
    for bad in ((-1, 1, 32, 8, 128), (1, 0, 32, 8, 128), (1, 1, 30, 8, 128), (1, 1, 32, 8, 96), (1, 1, 0, 1, 64)):
        assert f(*bad) == 0


def test_library_exports_the_header(lib):
    src = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "pard_serve.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(pard_[a-z_]+)\s*\(", src)))
    assert names == ["pard_adjust_logits", "pard_chunk_attention", "pard_chunk_attention_workspace_bytes", "pard_qk_norm_rope_quantized"]
    raw = ctypes.CDLL(lib._name)
    assert all(hasattr(raw, n) for n in names)


def test_calls_check_their_arguments_before_the_device():
    import torch

    from paper_2504_18583_gb300 import tree
    z = torch.zeros(2, 8)
    with pytest.raises(ValueError):
        tree.adjust_logits(z)
    with pytest.raises(ValueError):
        tree.chunk_attention(z, z, z, z, z, z)
    with pytest.raises(ValueError):
        tree.qk_norm_rope(z, 1, 1, z, z, z, z, None, k_scale=z, v_scale=z)
    with pytest.raises(ValueError):
        tree.chunk_attention_workspace(1, 1, 30, 8, 128)


def test_an_output_between_the_queries_rows_is_let_through(lib):
    """Refused for the workspace, which is looked at later."""
    edit = dict(q_stride=512 * 100, ws_bytes=4096)
    for out in (P + 2 * 512, P + 2 * 512 * 300 - 2 * 9 * 512, P + 2 * 512 * 800 + 2 * 512):
        assert call(lib, "pard_chunk_attention", CHUNK, out=out, **edit) == ARG
        assert b"workspace" in lib.pard_last_error()
    assert call(lib, "pard_chunk_attention", CHUNK, out=P + 2 * 512 * 300 - 2 * 9 * 512 + 16, **edit) == ARG
    assert b"over the queries" in lib.pard_last_error()


@pytest.mark.parametrize("T,batch,heads,group", [
    (262145, 1, 32, 1),   # one long prompt, blocks of 256 query vectors
    (49500, 49500, 1024, 1),  # a token a sequence, blocks of 128
    (70000, 3, 8, 4),
])
def test_the_limit_on_tiles_is_where_the_kernels_sums_end(lib, T, batch, heads, group):
    """A unit (a block of rows of a key/value head) counts its tiles of 128 keys and three more, and the sum over all
    units is held in 32 bits: page tables up to the last tile that fits are let through (and refused for the workspace,
    which is looked at later), one page more is refused for its size."""
    rows = 128 if T * group <= batch * 128 else 256
    units = (T * group // rows + batch) * heads
    tiles = (2 ** 31 - 1) // units - 3
    edit = dict(n_tokens=T, batch=batch, hq=heads * group, hkv=heads, q_stride=heads * group * 64, page_stride=heads * 16 * 64, ws_bytes=4096)
    assert units * (tiles + 3) < 2 ** 31 <= units * (tiles + 4)
    assert call(lib, "pard_chunk_attention", CHUNK, max_pages=tiles * 8, **edit) == ARG
    assert b"workspace" in lib.pard_last_error()
    assert call(lib, "pard_chunk_attention", CHUNK, max_pages=tiles * 8 + 1, **edit) == SHAPE
    assert b"2^31" in lib.pard_last_error()


@pytest.mark.parametrize("heads", [(32, 8, 128), (32, 32, 64), (64, 8, 128), (14, 2, 64), (64, 1, 64)])
def test_a_workspace_is_enough_for_fewer_tokens_and_sequences(lib, heads):
    """Many short sequences take blocks of 128 rows, fewer of them with as many tokens blocks of 256, whose partials are
    twice as large: the size for the former has to be enough for the latter."""
    f, sizes = lib.pard_chunk_attention_workspace_bytes, (1, 2, 4, 32, 33, 129, 256, 1000)
    for T in sizes:
        for batch in sizes:
            whole = f(T, batch, *heads)
            assert all(f(t, b, *heads) <= whole for t in sizes if t <= T for b in sizes if b <= batch)


# six rows of 100 floats (ADJUST)
@pytest.mark.parametrize("edit,over", [
    (dict(out=P + 4), True),                                   # an entry further
    (dict(z=P + 4, out=P), True),
    (dict(out=P + 5 * 400 + 396), True),                       # the last entry of all
    (dict(out=P + 6 * 400), False),
    (dict(z=P + 6 * 400, out=P), False),
    (dict(z=P + 5 * 400 + 396, out=P), True),
    (dict(out=P + 400), True),                                 # a row further
    (dict(out_stride=200), True),                              # the first row in place, the others not
    (dict(stride=200, out=P + 400, out_stride=200), False),    # rows between rows
    (dict(stride=200, out=P + 404, out_stride=200), True),
    (dict(stride=200, out=P + 396, out_stride=200), True),
    (dict(stride=200, out=P, out_stride=200), False),          # in place, rows apart
    (dict(stride=200, out=P + 800 * 3, out_stride=200), True),
    (dict(stride=300, out=P + 400, out_stride=150), True),     # rows 0 and 1 lie between rows, row 2 on one
    (dict(stride=400, out=P + 400, out_stride=800), False),    # at 400, 3600, 6800, ... against 0, 1600, 3200, ...
    (dict(batch=1, width=1, out=P + 400, out_stride=1000), False),
    (dict(batch=1, width=1, out=P, out_stride=1000), False),   # one row in place, whatever its stride
    (dict(batch=1, width=1, out=P + 396), True),
    (dict(dtype=0, out=P + 200), True),                        # 16-bit rows are half as long
    (dict(dtype=0, out=P + 1200), False),
])
def test_adjusted_logits_over_others(lib, edit, over):
    """An output that lies over other entries of the logits than its own is refused; in place, between the rows and apart
    from them it is not (and goes on to be refused for its tree, which is looked at later)."""
    args = {**ADJUST, "mask": None, **edit}
    size, rows = 4 if args["dtype"] == 2 else 2, args["batch"] * args["width"]
    of = {args["z"] + (r * args["stride"] + i) * size + b: (r, i) for r in range(rows) for i in range(100) for b in range(size)}
    hits = [of.get(args["out"] + (r * args["out_stride"] + i) * size + b, (r, i)) != (r, i) for r in range(rows) for i in range(100)
            for b in range(size)]
    hit = any(hits)
    assert hit == over
    assert call(lib, "pard_adjust_logits", args) == ARG
    assert (b"over the logits" if over else b"its mask") in lib.pard_last_error()
