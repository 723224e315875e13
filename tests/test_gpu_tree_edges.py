"""Edges of the tree operators that a wrong share, cut or rounding would show at:
against the 64-bit forms of test_gpu_tree.py, with its tolerances where no other
is derived here."""
import subprocess
import sys

import numpy as np
import pytest
import torch

from conftest import ROOT
from test_gpu_tree import (PAGE, ROUND, attention_reference, build_case, check_attention,  # noqa: F401
                           check_sample, dev, mask_of, rope_reference, tree)

pytestmark = pytest.mark.gpu


class Given:
    """Attention into outputs that start as NaN, with one workspace for all calls."""

    def __init__(self, tree, workspace):
        self.tree, self.workspace = tree, workspace

    def tree_attention(self, q, *args, **kw):
        out = torch.full(q.shape, float("nan"), dtype=q.dtype, device="cuda")
        return self.tree.tree_attention(q, *args, out=out, workspace=self.workspace, **kw)


@pytest.mark.parametrize("batch,Hkv,active", [
    (65, 1, {3: (60, 3)}), (65, 1, {64: (12, 1)}), (128, 1, {0: (148, 2)}), (65, 2, {40: (72, 5)}), (65, 4, {7: (34, 1)}),
    (65, 8, {0: (13, 2)}), (65, 8, {64: (15, 2)}), (128, 2, {5: (12, 1), 127: (20, 4)}), (400, 1, {399: (60, 2)}), (65, 1, {}),
])
def test_attention_large_batch_mostly_idle(tree, batch, Hkv, active):  # noqa: F811
    """More sequences than a CTA keeps at hand and less work than CTAs: most CTAs' ranges are empty, also in
    the middle of a unit.  active: sequence -> (tiles of 128 keys, nodes).  An ordinary call follows on the same
    workspace, whose arrival counts must be as it wants them."""
    lens, nodes = [0] * batch, [0] * batch
    for b, (tiles, n) in active.items():
        lens[b], nodes[b] = tiles * 128 - n - 3 * (b % 5), n
    given = Given(tree, tree.tree_attention_workspace(batch, 5, 4 * Hkv, Hkv, 64))
    for seed in (1, 2):
        check_attention(given, torch.bfloat16, 4 * Hkv, Hkv, 64, lens, nodes, 5, seed=seed)
        check_attention(given, torch.bfloat16, 4 * Hkv, Hkv, 64, [3000, 40], [5, 4], 5, seed=seed)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("k,m", [(0, 0.0), (3500, 0.0), (0, 1.0)])
def test_sample_empty_nucleus_among_ties(tree, dtype, k, m):  # noqa: F811
    """top_p = 0 (or below) where thousands of entries tie at the maximum and the lowest indices are not among
    them: the first of the tied is kept, alone."""
    V = 5003
    z = torch.zeros((5, V))
    z[0, 0] = float("-inf")
    z[1, :700] = -4.0
    z[2, :1500] = float("nan")
    z[3, :2000], z[3, 4000:] = -1e30, 3.0
    z[4, 1:3000] = 7.5
    R = len(z)
    for p in (0.0, -1.0, 1e-30):
        for T in (1.0, 1e-20):
            full = lambda v: np.full(R, v)  # noqa: E731
            assert check_sample(tree, z.to(dtype).cuda(), np.linspace(0, 0.99, R), full(T), full(k), full(p), full(m)) == R


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("Hq,Hkv,hd,nodes", [(8, 8, 128, 3), (8, 8, 64, 140)])
@pytest.mark.parametrize("hot", [0, 200, 639])
def test_attention_small_weights_add_up(tree, dtype, Hq, Hkv, hd, nodes, hot):  # noqa: F811
    """One key stands 5 to 20 nats above hundreds of others, and only the others' values are not zero: they share
    a mean, so that what is lost of each weight adds up.

    A weight is rounded to the type as 2^7 times its ratio to the largest so far: u of itself, or, among fp16's
    subnormals, 2^-25, which is 2^-32 of the largest's.  On top of u |o| + 2 u sum w |v| (test_gpu_tree.py) the
    output may then be off by 2^-32 sum |v|; bf16 has no subnormals there.  Scores of up to 20 are 32-bit sums of
    exact products: a weight's relative error of 20 * 2^-22 is far below u."""
    g = torch.Generator().manual_seed(hot + nodes)
    L = 640
    pages = -(-(L + nodes) // PAGE)
    k = torch.zeros((pages * PAGE, Hkv, hd))
    k[hot, :, 0] = 1.0
    v = 1024.0 * (1.0 + 0.25 * torch.rand((pages * PAGE, Hkv, hd), generator=g))
    v[hot] = 0.0
    q = torch.zeros((1, nodes, Hq, hd))
    nats = torch.tensor([5.0, 5.5, 10.0, 14.0, 17.0, 18.0, 19.0, 20.0])
    q[0, :, :, 0] = nats[:Hq] * hd ** 0.5
    q, k, v = q.to(dtype), k.to(dtype), v.to(dtype)
    paged = lambda x: x.view(pages, PAGE, Hkv, hd).transpose(1, 2).contiguous().cuda()  # noqa: E731
    mask = mask_of([[-1] + [0] * (nodes - 1)], [nodes], nodes)
    got = tree.tree_attention(q.cuda(), paged(k), paged(v), dev([list(range(pages))]), dev([L]), dev([nodes]),
                              torch.from_numpy(mask.view(np.int64)).cuda()).cpu()[0]
    sees = torch.ones((nodes, L + nodes), dtype=torch.bool)
    for i in range(nodes):
        for j in range(nodes):
            sees[i, L + j] = bool(int(mask[0, i, j // 64]) >> (j % 64) & 1)
    want, mag = attention_reference(q[0], k[:L + nodes], v[:L + nodes], sees, hd ** -0.5)
    tol = ROUND[dtype] * (want.abs() + 2 * mag)
    if dtype == torch.float16:
        tol = tol + 2.0 ** -32 * v[:L + nodes].double().abs().sum(0).amax() + 2.0 ** -24
    err = (got.double() - want).abs()
    assert (err <= tol).all(), float((err / tol).max())


@pytest.mark.parametrize("shared", [True, False])
@pytest.mark.parametrize("dtype,hd,lens,nodes,width", [
    (torch.bfloat16, 128, [2000, 77], [4, 5], 5),       # parts of units
    (torch.float16, 64, [300, 0, 9], [70, 64, 1], 70),  # two blocks of query vectors
    (torch.bfloat16, 64, [3000] + [7] * 69, [3] * 70, 4),  # ranges over many sequences
])
def test_attention_after_a_wait_ran_out(tree, shared, dtype, hd, lens, nodes, width):  # noqa: F811
    """The mark that a wait leaves in the workspace when it runs out, set by hand: every used node is NaN, call after
    call, and right again once the workspace has been zeroed."""
    B, Hq, Hkv = len(lens), 8, 4
    rs, g = np.random.RandomState(B), torch.Generator(device="cuda").manual_seed(B)
    parents, table, n_pages = build_case(rs, lens, nodes, width)
    mask = torch.from_numpy(mask_of(parents, nodes, width).view(np.int64)).cuda()
    kv = torch.randn((2, n_pages, Hkv, PAGE, hd), generator=g, device="cuda").to(dtype)
    q = torch.randn((B, width, Hq, hd), generator=g, device="cuda").to(dtype)
    workspace = None if shared else tree.tree_attention_workspace(B, width, Hq, Hkv, hd)
    call = lambda: tree.tree_attention(q, kv[0], kv[1], dev(table), dev(lens), dev(nodes), mask, workspace=workspace)  # noqa: E731
    want = call()
    used = torch.arange(width, device="cuda")[None] < dev(nodes)[:, None]
    assert torch.isfinite(want).all() and (want[used] != 0).any(-1).all()
    area = tree.shared_workspace() if shared else workspace
    area.view(torch.int32)[320] = 1  # behind two counts for each of up to 160 CTAs
    for _ in range(2):
        got = call()
        assert torch.isnan(got[used]).all() and (got[~used] == 0).all()
    area.zero_()
    assert torch.equal(call(), want)


@pytest.mark.parametrize("batch,most", [(385, 90), (1000, 20)])
def test_attention_more_sequences_than_threads(tree, batch, most):  # noqa: F811
    """The shares of more sequences than a CTA has threads are worked out in several steps, two rounds of them."""
    rs = np.random.RandomState(batch)
    lens, nodes = [int(x) for x in rs.randint(0, most, batch)], [int(x) for x in rs.randint(0, 5, batch)]
    lens[batch - 1], nodes[batch - 1] = 2000, 4
    check_attention(tree, torch.bfloat16, 4, 2, 64, lens, nodes, 4, seed=batch)


FIRST_CALLS = """
import sys
import torch
sys.path.insert(0, sys.argv[1])
from paper_2504_18583_gb300 import tree
g = torch.Generator(device="cuda").manual_seed(1)
z, u = torch.randn((3, 50000), generator=g, device="cuda"), torch.rand(3, generator=g, device="cuda")
q = torch.randn((1, 5, 8, 64), generator=g, device="cuda").bfloat16()
kv = torch.randn((2, 4, 2, 16, 64), generator=g, device="cuda").bfloat16()
i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")
table, ctx, nodes, mask = i32([[2, 0, 1, 3]]), i32([40]), i32([5]), torch.full((1, 5, 1), 31, device="cuda")
top_p = torch.full((3,), 0.9, device="cuda")
step = lambda: tree.sample(z, u, top_p=top_p) + (tree.tree_attention(q, kv[0], kv[1], table, ctx, nodes, mask),)
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    outs = step()
for _ in range(2):
    for x in outs:
        x.zero_()
    graph.replay()
    assert all(torch.equal(x, y) for x, y in zip(outs, step()))
print("same")
"""


def test_first_calls_of_a_process_inside_a_capture():
    """What a launch sets and asks once a device, it may do while a stream is being captured."""
    r = subprocess.run([sys.executable, "-c", FIRST_CALLS, ROOT], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip() == "same", r.stdout + r.stderr


def test_rotation_and_commit_past_32_bit_offsets(tree):  # noqa: F811
    """Pages that lie 1.5 GB apart: entry offsets pass 2^31 at the fourth page."""
    Hq, Hkv, hd, stride = 4, 2, 64, 768 * 1024 * 1024
    page = Hkv * PAGE * hd
    buf = torch.empty(3 * stride + 2 * page, dtype=torch.bfloat16, device="cuda")
    pool = buf.as_strided((1, 2, 4, Hkv, PAGE, hd), (8 * stride, page, stride, PAGE * hd, hd, 1))
    g = torch.Generator().manual_seed(4)
    start = torch.randn((1, 2, 4, Hkv, PAGE, hd), generator=g).to(torch.bfloat16)
    pool.copy_(start)
    # rows for every slot of the last page, and a few elsewhere
    slots = torch.tensor([3 * PAGE + i for i in range(PAGE)] + [5, 2 * PAGE + 1])
    T = len(slots)
    qkv = torch.randn((T, (Hq + 2 * Hkv) * hd), generator=g).to(torch.bfloat16)
    pos = torch.arange(T) + 7
    freq, _ = tree.rope_frequencies(hd)
    tree.qk_norm_rope(qkv.cuda(), Hq, Hkv, pos.to(torch.int32).cuda(), slots.cuda(), pool[0, 0], pool[0, 1], freq)
    x = qkv.view(T, -1, hd)
    keys = rope_reference(x[:, Hq:Hq + Hkv], None, 0.0, pos, freq.cpu(), hd, False, 1.0)
    got, want = pool.cpu(), start.clone()
    at = (slots // PAGE, slice(None), slots % PAGE)
    assert ((got[0, 0][at].double() - keys).abs() <= ROUND[torch.bfloat16] * keys.abs() + 2.0 ** -18 * keys.abs().amax(-1, keepdim=True)).all()
    want[0, 0][at], want[0, 1][at] = got[0, 0][at], x[:, Hq + Hkv:]
    assert torch.equal(got, want)
    # a path over the boundary between the second page of the table and the far one
    parents, tokens, sampled = [[-1, 0, 0, 2, 3, 3, 5]], [[0, 9, 1, 2, 9, 3, 4]], [[1, 0, 2, 3, 0, 4, 8]]
    table, ctx = [[1, 3, 0]], 14
    acc, emitted, new = tree.tree_commit(dev(sampled), dev(tokens), dev(parents), dev([7]), dev([ctx]), dev(table), pool)
    assert acc.tolist() == [4] and emitted.tolist() == [[1, 2, 3, 4, 8, -1, -1]] and new.tolist() == [ctx + 5]
    where = lambda i: (table[0][(ctx + i) // PAGE], (ctx + i) % PAGE)  # noqa: E731
    for j, i in enumerate([0, 2, 3, 5, 6]):
        (p, o), (sp, so) = where(j), where(i)
        want[:, :, p, :, o] = want[:, :, sp, :, so].clone()
    assert torch.equal(pool.cpu(), want)
