"""Tree attention joined from parts: infinities in nodes' values, and contexts up to
the largest, against test_gpu_tree.py's 64-bit forms, with its tolerances where no
other is derived here."""
import pytest
import torch

from test_gpu_tree import PAGE, ROUND, dev, run_attention, tree  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("Hq,Hkv,hd,n,ctx", [(8, 2, 64, 9, 6000), (64, 64, 128, 2, 3000), (128, 64, 64, 9, 3000), (16, 2, 64, 40, 6000)])
def test_infinities_of_nodes_with_far_lower_scores(tree, dtype, Hq, Hkv, hd, n, ctx):  # noqa: F811
    """Nodes' values in a part of the keys whose weights vanish (2^-173) beside another's: an infinity reaches the
    rows that see the node as what it is, whoever joins the parts (many, or two of which either may be the last)."""
    def edit(pool, table, q):
        q[..., 0] = 2.0 * hd ** 0.5
        for j in range(ctx + n):
            pool[table[0, j // PAGE], 0, :, j % PAGE, 0] = 30.0 if j < ctx // 2 else -30.0
        j = ctx + n // 2
        pool[table[0, j // PAGE], 1, :, j % PAGE, 7] = float("inf")
        pool[table[0, j // PAGE], 1, :, j % PAGE, hd - 1] = -float("inf")

    for seed in (1, 2):
        for _, got, want, tol, sees, v in run_attention(tree, dtype, Hq, Hkv, hd, [ctx], [n], n, seed=seed, edit=edit):
            sight = sees[:, ctx + n // 2]
            assert sight.any()
            assert torch.isposinf(got[sight][:, :, 7]).all() and torch.isneginf(got[sight][:, :, hd - 1]).all()
            fine = torch.ones_like(got, dtype=torch.bool)
            fine[sight, :, 7] = fine[sight, :, hd - 1] = False
            assert ((got.double() - want).abs() <= tol)[fine].all()


@pytest.mark.parametrize("keys", [2 ** 30, 128 * 8378391])  # the second: as many parts as CTAs, and no more
def test_the_longest_contexts(tree, keys):  # noqa: F811
    """Contexts up to 2^30, over a page table that names one page again and again: its 16 keys count alike.  A part's sums
    add up to 8 products a tile, each off by 2^-23 of the sum."""
    hd, n = 64, 1
    g = torch.Generator().manual_seed(1)
    pool, q = (torch.randn(shape, generator=g).bfloat16().cuda() for shape in ((3, 2, 1, PAGE, hd), (1, n, 1, hd)))
    table = torch.full((1, keys // PAGE), 1, dtype=torch.int32, device="cuda")
    out = torch.full_like(q, float("nan"))
    tree.tree_attention(q, pool[:, 0], pool[:, 1], table, dev([keys - n]), dev([n]), dev([[[1]]], torch.int64), out=out)
    k, v = pool[1, 0, 0].double(), pool[1, 1, 0].double()
    w = torch.softmax(q[0, 0].double() @ k.T / 8, -1)
    want, mag = w @ v, w @ v.abs()
    tol = ROUND[torch.bfloat16] * (want.abs() + 2 * mag) + keys / 128 / 100 * 8 * 2.0 ** -23 * mag
    assert ((out[0, 0].double() - want).abs() <= tol).all()
