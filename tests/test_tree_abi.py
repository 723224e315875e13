"""The tree operators' host side: every refusal comes before any CUDA call, so
these run without a GPU, with pointers that are never followed."""
import ctypes

import pytest

P = 0x10000  # 16-byte aligned, not null
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


PLAN = dict(parents=P, n_nodes=P, ctx=P, table=P, batch=2, width=9, max_pages=4, n_pages=8, mask=P, pos=P, slots=P, stream=None)
ROPE = dict(qkv=P, qkv_stride=12 * 64, dtype=0, n_tokens=3, hq=8, hkv=2, hd=64, qg=P, kg=None, eps=1e-6, pos=P, slots=P,
            freq=P, rot=64, inter=0, amp=1.0, q=P, q_stride=512, k=P, v=P, page_stride=2 * 16 * 64, n_pages=3, stream=None)
ATTN = dict(q=P, q_stride=512, dtype=1, batch=2, width=9, hq=8, hkv=2, hd=64, k=P, v=P, page_stride=2048, n_pages=3, table=P,
            max_pages=4, ctx=P, n=P, mask=P, scale=0.125, out=P, ws=P, ws_bytes=1 << 30, stream=None)
SAMPLE = dict(z=P, stride=100, dtype=2, rows=3, vocab=100, u=P, t=None, k=None, p=None, m=None, token=P, logprob=P, stream=None)
COMMIT = dict(sampled=P, tokens=P, parents=P, n=P, ctx=P, table=P, batch=2, width=9, max_pages=4, pool=P, ls=1 << 16, kvs=1 << 15,
              ps=2048, layers=2, hkv=2, hd=64, n_pages=3, acc=P, em=P, new=P, stream=None)


@pytest.mark.parametrize("name,good,edits", [
    ("pard_tree_plan", PLAN, [(dict(parents=None), ARG), (dict(slots=None), ARG), (dict(width=0), ARG), (dict(width=257), ARG),
                              (dict(batch=0), ARG), (dict(batch=65536), ARG), (dict(max_pages=0), ARG), (dict(n_pages=0), ARG)]),
    ("pard_qk_norm_rope", ROPE, [(dict(qkv=None), ARG), (dict(freq=None), ARG), (dict(dtype=2), SHAPE), (dict(hd=96), SHAPE),
                                 (dict(hd=256), SHAPE), (dict(rot=72), SHAPE), (dict(rot=128), SHAPE), (dict(rot=-16), SHAPE),
                                 (dict(qkv_stride=12 * 64 - 8), ARG), (dict(q_stride=504), ARG), (dict(qkv_stride=12 * 64 + 4), ARG),
                                 (dict(qkv=P + 2), ARG), (dict(v=P + 8), ARG), (dict(qg=P + 2), ARG), (dict(eps=-1.0), ARG),
                                 (dict(eps=float("nan")), ARG), (dict(page_stride=2047), SHAPE), (dict(page_stride=1024), SHAPE),
                                 (dict(n_tokens=-1), ARG), (dict(hkv=0), SHAPE), (dict(n_pages=0), SHAPE)]),
    ("pard_tree_attention", ATTN, [(dict(mask=None), ARG), (dict(ws=None), ARG), (dict(dtype=2), SHAPE), (dict(hq=7), SHAPE),
                                   (dict(hd=32), SHAPE), (dict(width=300), ARG), (dict(q_stride=500), ARG), (dict(q=P + 4), ARG),
                                   (dict(scale=float("inf")), ARG), (dict(ws_bytes=1000), ARG), (dict(page_stride=2052), SHAPE),
                                   (dict(batch=65535, max_pages=1 << 26), SHAPE), (dict(out=P + 2), ARG)]),
    ("pard_sample", SAMPLE, [(dict(z=None), ARG), (dict(u=None), ARG), (dict(token=None), ARG), (dict(dtype=3), SHAPE),
                             (dict(vocab=0), SHAPE), (dict(vocab=262145, stride=262145), SHAPE), (dict(stride=99), ARG),
                             (dict(rows=-1), ARG), (dict(z=P + 2), ARG)]),
    ("pard_tree_commit", COMMIT, [(dict(sampled=None), ARG), (dict(new=None), ARG), (dict(width=0), ARG), (dict(hd=80), SHAPE),
                                  (dict(layers=0), SHAPE), (dict(ls=7), ARG), (dict(pool=P + 2), ARG), (dict(ps=100), SHAPE)]),
])
def test_refusals_without_a_gpu(lib, name, good, edits):
    for edit, code in edits:
        assert call(lib, name, good, **edit) == code, (name, edit)
        assert lib.pard_last_error()


def test_empty_calls_do_nothing(lib):
    assert call(lib, "pard_sample", SAMPLE, rows=0, z=None) == 0
    assert call(lib, "pard_qk_norm_rope", ROPE, n_tokens=0, qkv=None) == 0


def test_workspace_sizes(lib):
    f = lib.pard_tree_attention_workspace_bytes
    assert f(1, 1, 32, 8, 128) > 0
    assert f(64, 256, 64, 8, 128) > f(1, 1, 32, 8, 128)  # two blocks of query vectors
    assert f(3, 9, 32, 8, 64) == f(50, 32, 32, 8, 64)    # by the blocks, not the batch
    for bad in ((0, 1, 32, 8, 128), (1, 257, 32, 8, 128), (1, 1, 30, 8, 128), (1, 1, 32, 8, 96), (1, 1, 0, 1, 64)):
        assert f(*bad) == 0


def test_module_needs_no_context():
    """The binding imports where the library is built; its calls check their arguments before the device."""
    import torch

    from paper_2504_18583_gb300 import tree
    z = torch.zeros(2, 8)
    with pytest.raises(ValueError):
        tree.sample(z, torch.zeros(2))
    with pytest.raises(ValueError):
        tree.tree_plan(None, None, None, None, 3)
    with pytest.raises(ValueError):
        tree.tree_plan(z.int(), z[:, 0].int(), z[:, 0].int(), z.int(), 3)
    assert ctypes.sizeof(ctypes.c_void_p) == 8
