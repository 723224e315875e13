"""Edges of the serving operators: against the 64-bit forms of test_gpu_serve.py,
with its tolerances where no other is derived here."""
import numpy as np
import pytest
import torch

from test_gpu_serve import BF, FP, PAGE, ROUND, Case, check_adjust, dev, tree, tree_mask, words_of  # noqa: F401

pytestmark = pytest.mark.gpu


# ---- chunk attention --------------------------------------------------------------
@pytest.mark.parametrize("eight", [False, True])
def test_a_workspace_of_a_larger_batch(tree, eight):  # noqa: F811
    """Made for many single tokens, used for a piece of a prompt of as many tokens and fewer, and for the batch again."""
    ws = tree.chunk_attention_workspace(256, 256, 8, 2, 128)
    for new, ctx in (([33], [700]), ([1] * 256, [40] * 256), ([256], [0]), ([200, 3], [9000, 4]), ([1], [3000])):
        Case(BF, 8, 2, 128, new, ctx, eight, seed=len(new)).check(tree, workspace=ws)
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


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("dtype", [BF, FP])
def test_a_prompt_in_pieces_row_by_row(tree, eight, dtype):  # noqa: F811
    """A prompt read whole, in uneven pieces and token by token: every output against 64 bits over the cache that was
    written.  In fp16 the tolerance tells a window that begins one key later, or one first token fewer, in every row (in
    bf16 its probabilities' rounding is as much as a key in some)."""
    Hq, Hkv, hd, T, window, sinks = 8, 2, 64, 333, 150, 4
    c = Case(dtype, Hq, Hkv, hd, [T, T], [0, 0], eight, seed=2)
    qkv = torch.randn((2 * T, (Hq + 2 * Hkv) * hd), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").to(dtype)
    freq, amp = tree.rope_frequencies(hd, 1e4)

    def read(pieces):
        if eight:
            c.k, c.v, c.ks, c.vs = tree.quantized_cache(c.n_pages, Hkv, hd)
        else:
            c.k, c.v = (torch.zeros((c.n_pages, Hkv, PAGE, hd), dtype=dtype, device="cuda") for _ in range(2))
        out, q, done = torch.empty_like(c.q), torch.empty_like(c.q), np.zeros(2, int)
        for new in pieces:
            rows = dev(np.concatenate([b * T + done[b] + np.arange(new[b]) for b in range(2)]), torch.int64)
            pos = [done[b] + np.arange(new[b]) for b in range(2)]
            slots = np.concatenate([c.table[b, p // PAGE] * PAGE + p % PAGE for b, p in enumerate(pos)])
            q[rows] = tree.qk_norm_rope(qkv[rows], Hq, Hkv, dev(np.concatenate(pos)), dev(slots, torch.int64), c.k, c.v, freq,
                                        amplitude=amp, k_scale=c.ks, v_scale=c.vs)
            out[rows] = tree.chunk_attention(q[rows], c.k, c.v, dev(c.table), dev(np.cumsum([0] + list(new))), dev(done), window=window,
                                             sinks=sinks, k_scale=c.ks, v_scale=c.vs)
            done += new
        assert (done == T).all()
        return out.double(), q

    for i, pieces in enumerate(([(T, T)], [(100, 1), (1, 231), (200, 1), (31, 1), (1, T - 234)], [(1, 2)] * 160 + [(T - 160, T - 320)])):
        got, c.q = read(pieces)
        if i == 0:
            if eight:
                c.ks, c.vs = c.ks.view(torch.uint8), c.vs.view(torch.uint8)
            want, tol = c.reference(window, sinks)
            late = torch.arange(2 * T, device="cuda") % T >= window + sinks
            for wrong in (c.reference(window - 1, sinks)[0], c.reference(window, sinks - 1)[0]) if dtype == FP else ():
                assert ((wrong - want).abs() > 2 * tol)[late].flatten(1).any(1).all()
        assert ((got - want).abs() <= tol).all(), float(((got - want).abs() / tol).max())


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("n,ctx", [(1, 2 ** 30 - 1), (1, 128 * (152 * 55188 - 1) - 1), (1, 128 * (152 * 54002 - 1) - 1), (300, 2 ** 30 - 300),
                                   (1, 128 * 8378391 - 1)])  # as many parts as CTAs, and no more
def test_the_longest_contexts(tree, eight, n, ctx):  # noqa: F811
    """Positions up to 2^30, over a page table that names one page again and again: all 16 keys count alike, but for the
    last few.  A part's sums add up to 8 products a tile, each off by 2^-23 of the sum."""
    c = Case(BF, 1, 1, 64, [n], [16], eight, seed=3)
    page, end = int(c.table[0, 0]), ctx + n
    c.ctx = [ctx]
    c.table = torch.full((1, -(-end // PAGE)), page, dtype=torch.int32, device="cuda")
    out = torch.full_like(c.q, float("nan"))
    got = tree.chunk_attention(c.q, c.k, c.v, c.table, dev(c.starts), dev(c.ctx), k_scale=c.ks, v_scale=c.vs, out=out)[:, 0].double()
    k, v = (c.values(w, [page])[0] for w in "kv")
    pos = torch.arange(ctx, end, device="cuda")[:, None]
    times = (pos - torch.arange(PAGE, device="cuda")) // PAGE + 1
    w = torch.exp((c.q[:, 0].double() @ k.T) / 8) * times
    w /= w.sum(1, keepdim=True)
    want, mag = w @ v, w @ v.abs()
    tol = ROUND[BF] * (want.abs() + 2 * mag) + end / 128 / 100 * 8 * 2.0 ** -23 * mag
    assert ((got - want).abs() <= tol).all(), float(((got - want).abs() / tol).max())


def test_a_unit_that_takes_longer_than_a_wait_may(tree):  # noqa: F811
    """8-bit caches, a sequence of 2^29 keys: the CTA that comes to the short one's heads has been at its first part for
    three seconds then, longer than a wait inside the kernel may last, and has many more parts after it."""
    heads, hd, keys = torch.cuda.get_device_properties(0).multi_processor_count, 64, 2 ** 29
    c = Case(BF, heads, heads, hd, [1, 1], [15, 5], True, seed=4)
    want, tol = c.reference()
    c.ctx = [keys - 1, 5]
    table = torch.zeros((2, keys // PAGE), dtype=torch.int32, device="cuda")
    table[0], table[1, 0] = int(c.table[0, 0]), int(c.table[1, 0])
    c.table = table
    got = tree.chunk_attention(c.q, c.k, c.v, c.table, dev(c.starts), dev(c.ctx), k_scale=c.ks, v_scale=c.vs,
                               out=torch.full_like(c.q, float("nan"))).double()
    assert ((got[1] - want[1]).abs() <= tol[1]).all()
    # the long one's sums pass what 32 bits tell apart: a weighted mean of its 16 values all the same
    v = c.values("v", [int(table[0, 0])])
    assert ((got[0] > 2 * v.amin(1) - 1) & (got[0] < 2 * v.amax(1) + 1)).all()


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


@pytest.mark.parametrize("grammar,branch,inplace", [(False, False, False), (True, False, True), (True, True, False), (False, True, True)])
@pytest.mark.parametrize("dtype,B,N,V,L", [
    (torch.float32, 600, 2, 4096, 900),   # slices of 4096: four pieces a thread; a CTA has both rows
    (BF, 64, 1, 128256, 8000),            # slices of 6752
    (FP, 64, 3, 128256, 6000),
    (torch.float32, 5, 29, 2048, 1500),   # rows shared out over CTAs
    (torch.float32, 1, 300, 700, 600),    # a CTA a row or two
])
def test_adjust_more_entries_than_threads(tree, dtype, B, N, V, L, grammar, branch, inplace):  # noqa: F811
    """Slices of which more than 256 entries change, so that threads take them in turns; long slices; several rows a CTA;
    in place too."""
    if branch and N > 256:
        branch = False
    rs = np.random.RandomState(V + N)
    z = (4 * torch.randn((B * N, V), generator=torch.Generator(device="cuda").manual_seed(V), device="cuda")).to(dtype)
    kw = dict(hist=rs.randint(-1, V + 1, (B, L)), hist_len=rs.randint(L - 50, L + 3, B), prompt_len=rs.randint(0, L, B),
              rep=rs.uniform(0.7, 1.5, B), freq=rs.uniform(-0.5, 0.5, B), pres=rs.uniform(-1, 1, B), ids=rs.randint(0, V, (B, 40)),
              bias=rs.uniform(-5, 5, (B, 40)), allowed=words_of(rs.rand(B * N, V) < 0.6) if grammar else None)
    if branch:
        kw.update(tokens=kw["hist"][:, :N] % V, mask=tree_mask(rs, B, N))  # a branch's tokens are in the history too
    if inplace:  # (check_adjust takes the values from z before the call)
        got = check_adjust(tree, z, N, out=z, **kw)
        assert got.data_ptr() == z.data_ptr()
    else:
        check_adjust(tree, z, N, **kw)
