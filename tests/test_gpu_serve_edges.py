"""Edges of the serving operators: against the 64-bit forms of test_gpu_serve.py,
with its tolerances where no other is derived here."""
import pytest
import torch

from test_gpu_serve import BF, FP, PAGE, Case, tree  # noqa: F401

pytestmark = pytest.mark.gpu


# ---- chunk attention --------------------------------------------------------------
@pytest.mark.parametrize("eight", [False, True])
def test_a_workspace_of_a_larger_batch(tree, eight):  # noqa: F811
    """Made for many single tokens, used for a piece of a prompt of as many tokens and fewer, and for the batch again."""
    ws = tree.chunk_attention_workspace(256, 256, 32, 8, 128)
    for new, ctx in (([33], [700]), ([1] * 256, [40] * 256), ([256], [0]), ([200, 3], [9000, 4]), ([1], [3000])):
        Case(BF, 32, 8, 128, new, ctx, eight, seed=len(new)).check(tree, workspace=ws)
    assert int(ws[:1296].sum()) == 0


def levels(c, low):
    """Scores of about +60, or -60 at positions that low() names, plus what the other entries give: 2^173 between the weights, more
    than the exponents of 32 bits hold beside the largest, and none of it matters to what an infinity is."""
    c.q[:, :, 0] = 2.0 * c.hd ** 0.5
    for b in range(len(c.new)):
        for pos in range(c.ctx[b] + c.new[b]):
            c.k[int(c.table[b, pos // PAGE]), :, pos % PAGE, 0] = -30.0 if low(pos) else 30.0


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("Hq,Hkv,hd,n", [
    (8, 2, 64, 20), (8, 2, 128, 2),   # a unit in many parts, of many rows and of few
    (128, 64, 64, 20), (64, 64, 128, 2),  # in two: either CTA may be the last
    (16, 4, 64, 100),                 # blocks of 256 rows
])
@pytest.mark.parametrize("where", ["last", "window"])
def test_infinities_in_a_part_of_far_lower_scores(tree, dtype, Hq, Hkv, hd, n, where):  # noqa: F811
    """Values that only some rows of a block see, in a part of the keys whose weights vanish beside another part's: they
    reach the rows that see them as what they are, whoever joins the parts.  The second block of 256 rows sees the first
    of them whole, so that it is multiplied by its weight: 2^-173 is 0 in 32 bits, and 0 times an infinity is NaN, so that
    either is right there."""
    ctx = 3000 if Hkv == 64 else 6000
    c = Case(dtype, Hq, Hkv, hd, [n], [ctx], seed=n + hd)
    window = 0 if where == "last" else ctx - ctx // 4
    if where == "last":
        levels(c, lambda pos: pos >= ctx // 2)
        at = [ctx + n // 2, ctx + n - 1]
    else:
        first = ctx - window + 1  # the first row's window begins here
        levels(c, lambda pos: pos < (first + ctx) // 2)
        at = [first, first + n // 2 - 1]
    for pos, x, col in zip(at, (float("inf"), float("nan")), (5, hd - 3)):
        c.v[int(c.table[0, pos // PAGE]), :, pos % PAGE, col] = x
        c.v[int(c.table[0, pos // PAGE]), :, pos % PAGE, 9] = -float("inf")
    want, tol = c.reference(window)
    either = torch.zeros_like(want, dtype=torch.bool)
    if where == "last" and n * Hq // Hkv > 256:
        either[256 * Hkv // Hq:, :, [5, 9]] = True
    assert torch.isinf(want[either]).all()
    for _ in range(5):
        got = c.call(tree, window, out=torch.full_like(c.q, 7.25)).double()
        assert not torch.isfinite(got[either]).any()
        odd = ~torch.isfinite(want) & ~either
        assert torch.equal(got[odd].nan_to_num(nan=1.0), want[odd].nan_to_num(nan=1.0))
        fine = torch.isfinite(want)
        assert ((got - want).abs() <= tol)[fine].all()


# ---- adjusted logits ------------------------------------------------------------------
def test_adjusted_logits_over_others_are_refused(tree):  # noqa: F811
    from paper_2504_18583_gb300.pard import PardError
    z = torch.randn((5, 240), device="cuda")
    kept, flat = z.clone(), z.view(-1)
    for at, out in ((z[:, :200], z[:, 1:201]), (z[1:, :200], z[:4, :200]), (flat[:200].view(1, 200), flat[199:399].view(1, 200)),
                    (z[:, :200], flat[:1000].view(5, 200))):
        with pytest.raises(PardError):
            tree.adjust_logits(at, out=out)
    assert torch.equal(z, kept)
    tree.adjust_logits(z[:, :120], out=z[:, 120:])  # beside each other
    assert torch.equal(z[:, 120:], kept[:, :120]) and torch.equal(z[:, :120], kept[:, :120])
