"""The tree decode step's operators against plain 64-bit implementations.

Tolerances, with u the output type's unit roundoff (2^-8 bf16, 2^-11 fp16):
rotated heads are computed in 32 bits and rounded once: u |y| plus 2^-18 of the
head's largest entry (sums of 128 squares and one rotation in 32 bits).
Attention rounds probabilities and the output: u |o| + 2 u sum_j w_j |v_j|, the
second u covering the scores' 32-bit products of up to 128 entries (relative
error of a weight below 2^-12 at the scores used).  Draws must be the
reference's unless u lies within 2^-20 of the boundary between two tokens
(weights are exact to 2^-23 each); log-probabilities within 2^-17 (1 + |lp|).
Whole numbers and moved rows are exact."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

ROUND = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
PAGE = 16


@pytest.fixture(scope="module")
def tree():
    from paper_2504_18583_gb300 import _build, tree
    _build.build()
    return tree


def dev(a, dtype=torch.int32):
    return torch.tensor(np.asarray(a), dtype=dtype, device="cuda")


def random_tree(rs, n):
    return [-1] + [int(rs.randint(max(0, i - 6), i)) for i in range(1, n)]


def ancestors(parents, i):
    out = set()
    while i >= 0:
        out.add(i)
        i = parents[i]
    return out


def build_case(rs, lens, nodes, width, extra=2):
    """Trees and a shuffled page table; unused page-table entries point outside the pool."""
    B = len(lens)
    parents = rs.randint(-5, 300, (B, width))
    for b, n in enumerate(nodes):
        parents[b, :n] = random_tree(rs, n) if n else []
    need = [-(-(l + n) // PAGE) for l, n in zip(lens, nodes)]
    order = rs.permutation(sum(need) + extra)
    P = max(max(need), 1) + 1
    table, at = np.full((B, P), 10 ** 6), 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return parents, table, len(order)


def mask_of(parents, nodes, width):
    W = -(-width // 64)
    m = np.zeros((len(nodes), width, W), np.uint64)
    for b, n in enumerate(nodes):
        for i in range(n):
            for j in ancestors(parents[b], i):
                m[b, i, j // 64] |= np.uint64(1) << np.uint64(j % 64)
    return m


# ---- plan -----------------------------------------------------------------------
@pytest.mark.parametrize("width,nodes", [(1, [1, 0]), (5, [5, 3, 1]), (64, [64, 63]), (65, [65, 64, 2]),
                                         (256, [256, 200, 0, 129])])
def test_plan(tree, width, nodes):
    rs = np.random.RandomState(width)
    lens = [int(x) for x in rs.randint(0, 70, len(nodes))]
    parents, table, n_pages = build_case(rs, lens, nodes, width)
    mask, pos, slots = tree.tree_plan(dev(parents), dev(nodes), dev(lens), dev(table), n_pages)
    want = mask_of(parents, nodes, width)
    assert np.array_equal(mask.cpu().numpy().view(np.uint64), want)
    for b, n in enumerate(nodes):
        for i in range(width):
            p, s = int(pos[b, i]), int(slots[b, i])
            if i >= n:
                assert (p, s) == (0, -1)
                continue
            assert p == lens[b] + len(ancestors(parents[b], i)) - 1
            at = lens[b] + i
            assert s == table[b, at // PAGE] * PAGE + at % PAGE


def test_plan_dead_nodes_and_missing_pages(tree):
    """A chain of 40 (the deepest tree of its size), a node whose parent follows
    it, its child, a parent below -1, and positions past the table."""
    parents = np.array([[-1] + list(range(39)), [-1, 0, 5, 2, -2, 1] + [0] * 34])
    mask, pos, slots = tree.tree_plan(dev(parents), dev([40, 6]), dev([10, 3]), dev([[7, 1], [900, 2]]), 8)
    m = mask.cpu().numpy().view(np.uint64)[:, :, 0]
    assert [int(x) for x in m[0]] == [(1 << (i + 1)) - 1 for i in range(40)]
    assert pos[0].tolist() == list(range(10, 50))
    want = [(7 if i < 16 else 1) * 16 + i % 16 if i < 32 else -1 for i in range(10, 50)]
    assert slots[0].tolist() == want
    assert [int(x) for x in m[1][:7]] == [1, 3, 0, 0, 0, 0b100011, 0]
    assert pos[1, :7].tolist() == [3, 4, 0, 0, 0, 5, 0]
    assert slots[1].tolist() == [-1] * 40  # page 900 is outside the pool


# ---- norm, rotation, cache write ---------------------------------------------------
def rope_reference(x, gain, eps, pos, freq, rot, interleaved, amp):
    y = x.double()
    if gain is not None:
        y = y / (y.square().mean(-1, keepdim=True) + eps).sqrt() * gain.double()
    ang = (pos.double()[:, None] * freq.double()[None])[:, None]
    c, s = amp * ang.cos(), amp * ang.sin()
    out = y.clone()
    if rot:
        ia, ib = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
        a, b = y[..., ia], y[..., ib]
        out[..., ia], out[..., ib] = a * c - b * s, a * s + b * c
    return out


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("Hq,Hkv,hd,rot,interleaved,norm,T,start", [
    (32, 8, 128, 128, False, True, 9, 512),
    (32, 8, 64, 64, False, True, 7, 131000),
    (64, 8, 128, 128, True, True, 3, 1000003),
    (8, 1, 128, 32, False, True, 33, 77),
    (4, 4, 64, 16, True, False, 5, 0),
    (3, 1, 64, 0, False, True, 2, 9),
    (5, 5, 128, 96, False, False, 400, 4000),
    (1, 1, 64, 48, False, True, 1, 2 ** 31 - 2),
])
def test_qk_norm_rope(tree, dtype, Hq, Hkv, hd, rot, interleaved, norm, T, start):
    g = torch.Generator().manual_seed(T * 7 + rot)
    cols = (Hq + 2 * Hkv) * hd
    wide = torch.randn((T, cols + 24), generator=g).to(dtype)
    if T > 1:
        wide[1] = 0  # a row without a norm
    buf = wide.cuda()
    qkv, x = buf[:, 8:8 + cols], wide[:, 8:8 + cols].view(T, -1, hd)
    pos = torch.arange(T) + start
    n_pages = T // PAGE + 2
    order = torch.randperm(n_pages * PAGE, generator=g)[:T]
    slots = order.clone()
    if T > 2:
        slots[2] = -1
        slots[-1] = n_pages * PAGE  # past the pool: not written
    pool = torch.full((n_pages, 2, Hkv, PAGE, hd), 7.0, dtype=dtype, device="cuda")  # keys and values of a page together
    freq, amp = (tree.rope_frequencies(rot, 500000.0, "yarn", 4.0, 8192, 1.0, 32.0) if rot else (None, 1.0))
    gains = [(1 + 0.3 * torch.randn(hd, generator=g)).to(dtype) if norm else None for _ in range(2)]
    q = tree.qk_norm_rope(qkv, Hq, Hkv, pos.to(torch.int32).cuda(), slots.cuda(), pool[:, 0], pool[:, 1], freq,
                          q_gain=None if not norm else gains[0].cuda(), k_gain=None if not norm else gains[1].cuda(),
                          eps=1e-5, interleaved=interleaved, amplitude=amp)
    f = torch.zeros(0) if freq is None else freq.cpu()
    rq = rope_reference(x[:, :Hq], gains[0], 1e-5, pos, f, rot, interleaved, amp)
    rk = rope_reference(x[:, Hq:Hq + Hkv], gains[1], 1e-5, pos, f, rot, interleaved, amp)

    def near(got, want):
        err = (got.double().cpu() - want).abs()
        tol = ROUND[dtype] * want.abs() + 2.0 ** -18 * want.abs().amax(-1, keepdim=True) + 2.0 ** -25
        assert (err <= tol).all(), float((err - tol).max())

    near(q, rq)
    got = pool.cpu()
    written = torch.zeros((n_pages, PAGE), dtype=torch.bool)
    for t in range(T):
        s = int(slots[t])
        if not 0 <= s < n_pages * PAGE:
            continue
        written[s // PAGE, s % PAGE] = True
        near(got[s // PAGE, 0, :, s % PAGE], rk[t])
        assert torch.equal(got[s // PAGE, 1, :, s % PAGE], x[t, Hq + Hkv:])
    left = got.permute(0, 3, 1, 2, 4)[~written]
    assert (left == 7.0).all()


def test_rope_frequencies(tree):
    base, amp = tree.rope_frequencies(64, 10000.0, device="cpu")
    assert amp == 1.0 and base[0] == 1.0 and math.isclose(float(base[1]), 10000.0 ** (-2 / 64), rel_tol=1e-6)
    lin, _ = tree.rope_frequencies(64, 10000.0, "linear", 8.0, device="cpu")
    assert torch.allclose(lin * 8, base, rtol=1e-6)
    ntk, _ = tree.rope_frequencies(64, 10000.0, "ntk", 8.0, device="cpu")
    assert ntk[0] == 1.0 and math.isclose(float(ntk[-1]) * 8, float(base[-1]), rel_tol=1e-5)
    for kind in ("parts", "yarn"):
        f, amp = tree.rope_frequencies(64, 10000.0, kind, 8.0, 8192, 1.0, 32.0, device="cpu")
        assert f[0] == base[0] and math.isclose(float(f[-1]) * 8, float(base[-1]), rel_tol=1e-6)
        ratio = f / base
        assert (ratio[1:] <= ratio[:-1] + 1e-7).all()
        assert math.isclose(amp, 0.1 * math.log(8) + 1 if kind == "yarn" else 1.0)
    with pytest.raises(ValueError):
        tree.rope_frequencies(64, 10000.0, "other", 8.0)


# ---- attention ------------------------------------------------------------------------
def attention_reference(q, k, v, sees, scale):
    """q [n, Hq, hd]; k, v [L, Hkv, hd]; sees [n, L].  Returns o and sum_j w_j |v_j|."""
    n, Hq, hd = q.shape
    group = Hq // k.shape[1]
    o, a = torch.zeros(q.shape, dtype=torch.float64), torch.zeros(q.shape, dtype=torch.float64)
    if not k.shape[0]:
        return o, a
    for h in range(Hq):
        s = scale * (q[:, h].double() @ k[:, h // group].double().T)
        s = s.masked_fill(~sees, float("-inf"))
        some = sees.any(1)
        w = torch.zeros_like(s)
        w[some] = torch.softmax(s[some], -1)
        vv = v[:, h // group].double()
        vis = torch.where(torch.isfinite(vv), vv, 0.0)
        o[:, h], a[:, h] = w @ vis, w @ vis.abs()
    return o, a


def run_attention(tree, dtype, Hq, Hkv, hd, lens, nodes, width, seed, mask=None, spread=1.0, poison=True, scale=None,
                  edit=None, splitless=False):
    rs = np.random.RandomState(seed)
    g = torch.Generator().manual_seed(seed)
    parents, table, n_pages = build_case(rs, lens, nodes, width)
    if mask is None:
        mask = mask_of(parents, nodes, width)
    B = len(lens)
    pool = torch.randn((n_pages, 2, Hkv, PAGE, hd), generator=g)
    q = spread * torch.randn((B, width, Hq + 3, hd), generator=g)
    used = torch.zeros((n_pages, PAGE), dtype=torch.bool)
    for b in range(B):
        for j in range(lens[b] + nodes[b]):
            used[table[b, j // PAGE], j % PAGE] = True
    if poison:  # what lies past a sequence's keys is nobody's
        pool.permute(0, 3, 1, 2, 4)[~used] = float("nan")
        for b in range(B):
            q[b, nodes[b]:] = float("nan")
    pool, q = pool.to(dtype), q.to(dtype)
    if edit:
        edit(pool, table, q)
    dp, dq = pool.cuda(), q.cuda()
    out = tree.tree_attention(dq[:, :, :Hq], dp[:, 0], dp[:, 1], dev(table), dev(lens), dev(nodes),
                              torch.from_numpy(mask.view(np.int64)).cuda(), scale=scale)
    again = tree.tree_attention(dq[:, :, :Hq], dp[:, 0], dp[:, 1], dev(table), dev(lens), dev(nodes),
                                torch.from_numpy(mask.view(np.int64)).cuda(), scale=scale)
    got = out.cpu()
    assert torch.equal(got.view(torch.int16), again.cpu().view(torch.int16))
    for b in range(B):
        L, n = lens[b], nodes[b]
        assert (got[b, n:] == 0).all()
        idx = [(table[b, j // PAGE], j % PAGE) for j in range(L + n)]
        pg, of = [i[0] for i in idx], [i[1] for i in idx]
        k, v = pool[pg, 0][torch.arange(L + n), :, of], pool[pg, 1][torch.arange(L + n), :, of]
        sees = torch.ones((n, L + n), dtype=torch.bool)
        for i in range(n):
            for j in range(n):
                sees[i, L + j] = bool(int(mask[b, i, j // 64]) >> (j % 64) & 1)
        want, mag = attention_reference(q[b, :n, :Hq], k, v, sees, hd ** -0.5 if scale is None else scale)
        err = (got[b, :n].double() - want).abs()
        tol = ROUND[dtype] * (want.abs() + 2 * mag) + 2.0 ** -24
        bad = ~(err <= tol)
        if edit is None:
            assert not bad.any(), (b, float((err / tol).max()), int(bad.sum()))
        yield b, got[b, :n], want, tol, sees, v


def check_attention(*args, **kw):
    for _ in run_attention(*args, **kw):
        pass


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("Hq,Hkv,hd", [(32, 8, 128), (32, 8, 64), (16, 2, 128), (7, 7, 64), (5, 1, 128)])
@pytest.mark.parametrize("lens,nodes,width", [
    ([512], [1], 1),
    ([0, 1, 15, 16, 17], [1, 3, 0, 5, 4], 5),
    ([127, 128, 129, 1000], [13, 29, 1, 20], 29),
    ([300, 77], [64, 41], 64),
])
def test_attention(tree, dtype, Hq, Hkv, hd, lens, nodes, width):
    check_attention(tree, dtype, Hq, Hkv, hd, lens, nodes, width, seed=len(lens) * 100 + width)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("hd", [64, 128])
def test_attention_widest_tree_and_long_context(tree, dtype, hd):
    check_attention(tree, dtype, 8, 2, hd, [63, 2500], [256, 130], 256, seed=3)
    check_attention(tree, dtype, 8, 2, hd, [20011, 3], [3, 2], 3, seed=4, spread=2.0)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("Hq,Hkv,hd,width", [(32, 32, 128, 3), (32, 32, 64, 5), (64, 16, 128, 40), (96, 24, 64, 33)])
def test_attention_many_tiles_a_cta(tree, dtype, Hq, Hkv, hd, width):
    """Ranges of a dozen tiles and more, of several units: every stage of the ring is used again and again."""
    check_attention(tree, dtype, Hq, Hkv, hd, [5000, 1777, 3, 2900], [width, width - 1, width, 2], width, seed=width)


def test_attention_many_short_sequences(tree):
    rs = np.random.RandomState(8)
    lens, nodes = [int(x) for x in rs.randint(0, 200, 70)], [int(x) for x in rs.randint(0, 10, 70)]
    check_attention(tree, torch.bfloat16, 8, 4, 128, lens, nodes, 9, seed=9)


def test_attention_peaked_scores(tree):
    """Scores spread over hundreds: the running maximum moves far, most weights vanish."""
    check_attention(tree, torch.bfloat16, 8, 2, 128, [700, 1500], [9, 4], 9, seed=5, spread=30.0)
    check_attention(tree, torch.float16, 8, 2, 64, [700, 1500], [9, 4], 9, seed=6, spread=30.0, scale=-0.2)


@pytest.mark.parametrize("hd", [64, 128])
def test_attention_rows_that_see_nothing(tree, hd):
    """Without a context, rows of an all-zero mask are empty: zero, not NaN; bits past the nodes are ignored."""
    mask = np.zeros((2, 6, 1), np.uint64)
    mask[0, 1, 0], mask[0, 3, 0], mask[1, 0, 0] = 0b10, 0b101, 0xFFFFFFFFFFFFFFFF
    check_attention(tree, torch.bfloat16, 8, 2, hd, [0, 0], [5, 2], 6, seed=11, mask=mask)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_attention_nonfinite_in_masked_nodes(tree, dtype):
    """One branch's keys and values hold NaN and infinities: only the rows that see it are touched."""
    def edit(pool, table, q):
        for j, val in ((203, float("nan")), (204, float("inf"))):
            pool[table[0, j // PAGE], 0, :, j % PAGE] = float("nan")
            pool[table[0, j // PAGE], 1, :, j % PAGE, 5] = val
    mask = np.zeros((1, 8, 1), np.uint64)
    for i in range(8):
        mask[0, i, 0] = np.uint64(1 << i | 1)
    for _, got, want, tol, sees, v in run_attention(tree, dtype, 4, 2, 128, [200], [8], 8, seed=12, mask=mask,
                                                    edit=edit):
        clean = [0, 1, 2, 5, 6, 7]
        assert ((got[clean].double() - want[clean]).abs() <= tol[clean]).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_attention_nonfinite_value_reaches_who_sees_it(tree, dtype):
    """Infinite and NaN entries of one node's value show in the rows that see the node, in their columns only."""
    def edit(pool, table, q):
        j = 203
        pool[table[0, j // PAGE], 1, :, j % PAGE, 5] = float("inf")
        pool[table[0, j // PAGE], 1, :, j % PAGE, 9] = float("nan")
        pool[table[0, j // PAGE], 1, :, j % PAGE, 11] = float("-inf")
    for _, got, want, tol, sees, v in run_attention(tree, dtype, 4, 2, 128, [200], [8], 8, seed=13, edit=edit):
        for i in range(8):
            row = got[i].double()
            cols = [c for c in range(128) if c not in (5, 9, 11)]
            assert ((row[:, cols] - want[i][:, cols]).abs() <= tol[i][:, cols]).all()
            if sees[i, 203]:
                assert torch.isposinf(row[:, 5]).all() and torch.isnan(row[:, 9]).all() and torch.isneginf(row[:, 11]).all()
            else:
                assert torch.isfinite(row).all()


def test_attention_cache_past_32_bit_offsets(tree):
    """Pages that lie 1.5 GB apart: entry offsets pass 2^31 at the fourth page."""
    Hkv, hd, stride = 2, 64, 768 * 1024 * 1024
    buf = torch.empty(3 * stride + 2 * PAGE * hd * Hkv, dtype=torch.bfloat16, device="cuda")
    g = torch.Generator().manual_seed(2)
    caches = []
    for part in range(2):
        view = buf.as_strided((4, Hkv, PAGE, hd), (stride, PAGE * hd, hd, 1), part * PAGE * hd * Hkv)
        data = torch.randn((4, Hkv, PAGE, hd), generator=g).to(torch.bfloat16)
        view.copy_(data)
        caches.append((view, data))
    q = torch.randn((1, 3, 4, hd), generator=g).to(torch.bfloat16)
    mask = np.array([[[1], [3], [5]]], np.uint64)
    table = [[3, 0, 2, 1]]
    out = tree.tree_attention(q.cuda(), caches[0][0], caches[1][0], dev(table), dev([60]), dev([3]),
                              torch.from_numpy(mask.view(np.int64)).cuda()).cpu()
    k, v = (c[1][table[0]].permute(0, 2, 1, 3).reshape(64, Hkv, hd)[:63] for c in caches)
    sees = torch.ones((3, 63), dtype=torch.bool)
    sees[:, 60:] = torch.tensor([[1, 0, 0], [1, 1, 0], [1, 0, 1]], dtype=torch.bool)
    want, mag = attention_reference(q[0], k, v, sees, hd ** -0.5)
    assert ((out[0].double() - want).abs() <= 2.0 ** -8 * (want.abs() + 2 * mag)).all()


@pytest.mark.parametrize("dtype,hd,width", [(torch.bfloat16, 128, 5), (torch.float16, 64, 200), (torch.float16, 128, 140)])
def test_attention_units_of_two_parts(tree, dtype, hd, width):
    """As many units as half of the CTAs and contexts to match: two CTAs share each, and whichever is last joins them.
    One node's values hold infinities: they reach those who see it whoever joins."""
    edit_at = 2400 + 1

    def edit(pool, table, q):
        pool[table[0, edit_at // PAGE], 1, :, edit_at % PAGE, 7] = float("inf")

    check_attention(tree, dtype, 70, 70, hd, [2400], [width], width, seed=width)
    for _, got, want, tol, sees, v in run_attention(tree, dtype, 70, 70, hd, [2400], [width], width, seed=width, edit=edit):
        sight = sees[:, edit_at]
        assert torch.isposinf(got[sight][:, :, 7]).all() and torch.isfinite(got[~sight]).all()
        cols = [c for c in range(hd) if c != 7]
        assert ((got.double() - want).abs() <= tol)[:, :, cols].all()


def test_attention_output_off_32_bytes(tree):
    """An output that is 16-byte aligned and no more, through the C call; bytes around it stay as they were."""
    from paper_2504_18583_gb300 import pard
    lib = pard.lib()
    B, N, Hq, Hkv, hd = 2, 6, 8, 2, 128
    g = torch.Generator(device="cuda").manual_seed(3)
    pool = torch.randn((12, 2, Hkv, PAGE, hd), generator=g, device="cuda").to(torch.bfloat16)
    q = torch.randn((B, N, Hq, hd), generator=g, device="cuda").to(torch.bfloat16)
    table, lens, nodes = dev([[0, 3, 5, 7, 9], [1, 2, 4, 6, 8]]), dev([60, 31]), dev([6, 4])
    mask = torch.ones((B, N, 1), dtype=torch.int64, device="cuda")
    want = tree.tree_attention(q, pool[:, 0], pool[:, 1], table, lens, nodes, mask)
    buf = torch.full((want.numel() + 32,), 7.0, dtype=torch.bfloat16, device="cuda")
    assert buf.data_ptr() % 32 == 0
    size = lib.pard_tree_attention_workspace_bytes(B, N, Hq, Hkv, hd)
    work = torch.zeros(size, dtype=torch.uint8, device="cuda")
    ptr = lambda t: t.data_ptr()  # noqa: E731
    status = lib.pard_tree_attention(ptr(q), Hq * hd, 0, B, N, Hq, Hkv, hd, ptr(pool), ptr(pool[:, 1]), pool.stride(0), 12,
                                     ptr(table), 5, ptr(lens), ptr(nodes), ptr(mask), hd ** -0.5, ptr(buf) + 16, ptr(work),
                                     size, torch.cuda.current_stream().cuda_stream)
    assert status == 0
    assert torch.equal(buf[8:-24].view_as(want), want)
    assert (buf[:8] == 7).all() and (buf[-24:] == 7).all()


def test_attention_on_another_stream(tree):
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        check_attention(tree, torch.bfloat16, 8, 2, 128, [333, 40], [7, 5], 7, seed=21)


# ---- sampling -------------------------------------------------------------------------
def sample_reference(z, T, k, p, m):
    """Kept indices in index order and their weights, in 64 bits."""
    z = np.where(np.isnan(z), -np.inf, z.astype(np.float64))
    order = np.lexsort((np.arange(len(z)), -z))
    with np.errstate(invalid="ignore"):
        w = np.exp(np.where(z == z.max(), 0.0, (z - z.max()) / T))
    if k > 0:
        order = order[:k]
    before = np.cumsum(w[order]) - w[order]
    keep = (before < p * w[order].sum()) & (w[order] >= m)
    keep[0] = True
    kept = np.sort(order[keep])
    return kept, w[kept]


def check_sample(tree, z, u, T, k, p, m):
    """z: device logits [R, V]; the rest numpy arrays [R]."""
    token, logp = tree.sample(z, dev(u, torch.float32), dev(T, torch.float32), dev(k), dev(p, torch.float32),
                              dev(m, torch.float32))
    zc = z.float().cpu().numpy()
    token, logp = token.cpu().numpy(), logp.cpu().numpy()
    f32 = lambda a: np.asarray(a, np.float32).astype(np.float64)  # noqa: E731
    u, T, p, m = f32(u), f32(T), f32(p), f32(m)
    exact = 0
    for r in range(len(zc)):
        row = np.where(np.isnan(zc[r]), -np.inf, zc[r])
        if row.max() == -np.inf:
            assert token[r] == -1 and logp[r] == -np.inf
            continue
        if T[r] <= 0:
            assert token[r] == int(np.argmax(row)) and logp[r] == 0
            continue
        kept, w = sample_reference(zc[r], T[r], int(k[r]), p[r], m[r])
        cum = np.cumsum(w) / w.sum()
        i = min(int(np.searchsorted(cum, u[r], side="right")), len(kept) - 1)
        if token[r] != kept[i]:
            assert token[r] in kept, (r, token[r])
            j = int(np.searchsorted(kept, token[r]))
            lo, hi = min(i, j), max(i, j)
            assert abs(cum[lo] - u[r]) < 2.0 ** -20 and cum[hi - 1] - cum[lo] < 2.0 ** -20, (r, token[r], kept[i])
            i = j
        else:
            exact += 1
        want = -math.log1p((w.sum() - w[i]) / w[i])
        assert abs(logp[r] - want) <= 2.0 ** -17 * (1 + abs(want)), (r, logp[r], want)
    return exact


def cuts(rs, R, mode):
    k = np.where(rs.rand(R) < 0.5, rs.randint(1, 300, R), 0) if "k" in mode else np.zeros(R, int)
    p = rs.uniform(0.3, 0.999, R) if "p" in mode else np.ones(R)
    m = rs.uniform(0.0, 0.3, R) if "m" in mode else np.zeros(R)
    return k, p, m


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("V", [1, 2, 37, 2048, 4099, 32003, 128256, 262144])
@pytest.mark.parametrize("mode", ["", "k", "p", "m", "kpm"])
def test_sample(tree, dtype, V, mode):
    rs = np.random.RandomState(V % 1000 + len(mode))
    R = 6
    g = torch.Generator().manual_seed(V)
    wide = torch.randn((R, V + 3), generator=g) * 2.5
    z = wide.to(dtype).cuda()[:, 1:V + 1]  # rows that start and end off any boundary
    k, p, m = cuts(rs, R, mode)
    T = rs.uniform(0.3, 1.6, R)
    T[0] = 0.0
    exact = check_sample(tree, z, rs.rand(R), T, k, p, m)
    assert exact >= R - 2


@pytest.mark.parametrize("V", [5000, 128256])
def test_sample_flat_and_tied_rows(tree, V):
    """All entries equal, two values only, a few distinct ones: cuts fall inside runs of ties."""
    rs = np.random.RandomState(7)
    z = np.zeros((6, V), np.float32)
    z[1, ::3] = 1.0
    z[2] = np.round(rs.randn(V) * 2) / 2
    z[3] = rs.randint(0, 2, V) * 40.0
    z[4] = 15 + np.round(rs.randn(V) * 4) / 8
    z[5] = -3.0
    for T in (1.0, 1e-3, 1e8):
        for k, p, m in ((0, 0.5, 0.0), (V // 3, 1.0, 0.0), (3000, 0.9, 0.0), (4000, 0.37, 0.2), (1, 0.9, 0.0), (0, 1.0, 1.0)):
            R = len(z)
            check_sample(tree, dev(z, torch.float32), rs.rand(R), np.full(R, T), np.full(R, k), np.full(R, p), np.full(R, m))


@pytest.mark.parametrize("dtype,V", [(torch.float32, 128256), (torch.float32, 20011), (torch.bfloat16, 50257), (torch.float16, 130001)])
def test_sample_wide_cuts_and_many_rows(tree, dtype, V):
    """Cuts in flat, rounded, heavy-tailed and peaked rows, where thousands of entries lie near them; a row's draw
    does not depend on how many rows there are (and with them how many CTAs share one)."""
    rs = np.random.RandomState(V % 997)
    g = torch.Generator().manual_seed(V)
    rows, k, p, m, T = [], [], [], [], []
    for kind in range(8):
        x = torch.randn(V, generator=g)
        z = [x * 0.05, x * 0.8, x * 3, torch.round(x * 8) / 8, torch.round(x * 2) / 64, -x.abs().pow(3), x.abs().sqrt() * 6,
             torch.where(torch.rand(V, generator=g) < 0.001, x + 9, x)][kind]
        for kk, pp, mm in ((0, 0.9, 0.0), (0, 0.999, 0.0), (0, 0.03, 0.0), (0, 0.97, 0.02), (257, 1.0, 0.0), (1500, 0.98, 0.0)):
            rows.append(z)
            k.append(kk), p.append(pp), m.append(mm), T.append(rs.uniform(0.5, 1.4))
    z = torch.stack(rows).to(dtype).cuda()
    u, k, p, m, T = rs.rand(len(rows)), np.array(k), np.array(p), np.array(m), np.array(T)
    assert check_sample(tree, z, u, T, k, p, m) >= len(rows) - 4
    f = lambda a: dev(a, torch.float32)  # noqa: E731
    few = [tree.sample(z[i:i + 6], f(u[i:i + 6]), f(T[i:i + 6]), dev(k[i:i + 6]), f(p[i:i + 6]), f(m[i:i + 6])) for i in range(0, 48, 6)]
    many = tree.sample(z.repeat(8, 1), f(np.tile(u, 8)), f(np.tile(T, 8)), dev(np.tile(k, 8)), f(np.tile(p, 8)), f(np.tile(m, 8)))
    for i in range(2):
        assert torch.equal(many[i], torch.cat([x[i] for x in few]).repeat(8))


def test_sample_masked_and_nonfinite_rows(tree):
    """-inf, NaN, +inf and the type's lowest value; rows without any entry."""
    V = 3001
    g = torch.Generator().manual_seed(1)
    z = torch.randn((9, V), generator=g)
    z[0] = float("-inf")
    z[1] = float("nan")
    z[2, 1:] = float("-inf")
    z[3, ::2] = float("nan")
    z[4, 7] = z[4, 2900] = float("inf")
    z[5, 100:] = torch.finfo(torch.float32).min
    z[6] = torch.finfo(torch.float32).min
    z[7, :2000] = float("-inf")
    z[8] = -1e30 * torch.rand(V, generator=g)
    R = len(z)
    rs = np.random.RandomState(3)
    for k, p, m in ((0, 1.0, 0.0), (50, 0.9, 0.01), (0, 0.9, 0.0), (2500, 1.0, 0.0), (2500, 0.99, 0.0)):
        for T in (1.0, 0.0):
            check_sample(tree, z.cuda(), rs.rand(R), np.full(R, T), np.full(R, k), np.full(R, p), np.full(R, m))


def test_sample_ends_of_the_unit_interval(tree):
    """u = 0 draws the first kept entry, the largest u below 1 the last; p = 0 keeps one."""
    V = 1000
    z = torch.zeros((4, V), device="cuda")
    z[:, 10] = 1.0
    u = np.array([0.0, 1 - 2.0 ** -24, 0.0, 0.7])
    token, _ = tree.sample(z, dev(u, torch.float32), top_p=dev([1, 1, 0, 0], torch.float32))
    assert token.tolist() == [0, V - 1, 10, 10]


def test_sample_follows_the_distribution(tree):
    """200000 draws from one row of eight entries: each frequency within five standard deviations."""
    z = torch.tensor([0.0, 1.0, -1.0, 2.0, 0.5, -3.0, 1.5, 0.0], device="cuda")
    n = 200000
    u = torch.rand(n, generator=torch.Generator(device="cuda").manual_seed(4), device="cuda")
    token, logp = tree.sample(z.repeat(n, 1), u)
    p = torch.softmax(z.double(), 0).cpu()
    freq = torch.bincount(token.long(), minlength=8).double().cpu() / n
    assert ((freq - p).abs() <= 5 * (p * (1 - p) / n).sqrt()).all()
    assert torch.allclose(logp.double().cpu(), p.log()[token.long().cpu()], atol=2.0 ** -16)


# ---- commit -----------------------------------------------------------------------------
def walk(parents, tokens, sampled, n):
    if n == 0:
        return []
    path = [0]
    while True:
        kids = [c for c in range(n) if parents[c] == path[-1] and c > path[-1] and tokens[c] == sampled[path[-1]] >= 0]
        if not kids:
            return path
        path.append(kids[0])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("Hkv,hd,L,lens,nodes,width", [
    (8, 128, 3, [30, 0, 16, 7], [29, 5, 1, 0], 29),
    (2, 64, 1, [100], [256], 256),
    (5, 64, 2, [15, 31, 47], [64, 64, 33], 64),
])
def test_commit(tree, dtype, Hkv, hd, L, lens, nodes, width):
    rs = np.random.RandomState(width)
    parents, table, n_pages = build_case(rs, lens, nodes, width)
    B = len(lens)
    tokens, sampled = rs.randint(0, 3, (B, width)), rs.randint(-1, 3, (B, width))  # few tokens: twins among children
    if width == 256:  # a long path: the chain 0, 2, 3, 4, ...
        parents[0, :256] = [-1, 0, 0] + list(range(2, 255))
        tokens[0], sampled[0] = 1, 1
        tokens[0, 1] = 2
    pool = torch.randn((2, L, n_pages, Hkv, PAGE, hd), generator=torch.Generator().manual_seed(width)).to(dtype)
    want = pool.permute(1, 0, 2, 3, 4, 5).clone()
    dpool = pool.cuda().permute(1, 0, 2, 3, 4, 5)  # keys of all layers, then values
    acc, em, new = tree.tree_commit(dev(sampled), dev(tokens), dev(parents), dev(nodes), dev(lens), dev(table), dpool)
    for b in range(B):
        path = walk(parents[b], tokens[b], sampled[b], nodes[b])
        assert int(acc[b]) == max(0, len(path) - 1) and int(new[b]) == lens[b] + len(path)
        assert em[b].tolist() == [int(sampled[b, i]) for i in path] + [-1] * (width - len(path))
        for j, i in enumerate(path):
            s, d = lens[b] + i, lens[b] + j
            want[:, :, table[b, d // PAGE], :, d % PAGE] = want[:, :, table[b, s // PAGE], :, s % PAGE].clone()
    assert torch.equal(dpool.cpu(), want)


# ---- refusals ---------------------------------------------------------------------------
def test_refusals(tree):
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
    z = torch.zeros((2, 8), device="cuda")
    u = torch.zeros(2, device="cuda")
    from paper_2504_18583_gb300.pard import PardError
    with pytest.raises(ValueError):
        tree.sample(z.cpu(), u)
    with pytest.raises(ValueError):
        tree.sample(z.double(), u)
    with pytest.raises(ValueError):
        tree.sample(z, u[:1])
    with pytest.raises(ValueError):
        tree.sample(z, u, top_k=u)
    with pytest.raises(PardError):
        tree.sample(torch.zeros((1, 262145), device="cuda"), u[:1])
    with pytest.raises(PardError):
        tree.tree_plan(i32(1, 257), i32(1), i32(1), i32(1, 4), 4)
    with pytest.raises(ValueError):
        tree.tree_plan(i32(1, 7), i32(2), i32(1), i32(1, 4), 4)
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    mask = torch.zeros((1, 2, 1), dtype=torch.int64, device="cuda")
    ok = (bf(1, 2, 4, 64), bf(3, 2, 16, 64), bf(3, 2, 16, 64), i32(1, 4), i32(1), i32(1), mask)
    tree.tree_attention(*ok)
    for at, bad in ((0, bf(1, 2, 3, 64)), (0, bf(1, 2, 4, 64).float()), (1, bf(3, 2, 8, 64)), (2, bf(3, 2, 16, 128)),
                    (3, i32(1, 4).long()), (6, mask[:, :1]), (0, bf(1, 2, 4, 72)[..., :64])):
        args = list(ok)
        args[at] = bad
        with pytest.raises((ValueError, PardError)):
            tree.tree_attention(*args)
    odd = (bf(1, 2, 4, 96), bf(3, 2, 16, 96), bf(3, 2, 16, 96)) + ok[3:]
    with pytest.raises((ValueError, PardError)):
        tree.tree_attention(*odd)
    with pytest.raises(PardError):
        tree.tree_attention(*ok, scale=float("nan"))
    f = torch.zeros(4, device="cuda")
    with pytest.raises(PardError):  # 8 rotated entries
        tree.qk_norm_rope(bf(3, 8 * 64), 4, 2, i32(3), i32(3).long(), bf(3, 2, 16, 64), bf(3, 2, 16, 64), f)
    with pytest.raises(ValueError):
        tree.qk_norm_rope(bf(3, 7 * 64), 4, 2, i32(3), i32(3).long(), bf(3, 2, 16, 64), bf(3, 2, 16, 64), None)
    with pytest.raises(PardError):  # rows off 16 bytes
        tree.qk_norm_rope(bf(3, 8 * 64 + 8)[:, 1:513], 4, 2, i32(3), i32(3).long(), bf(3, 2, 16, 64), bf(3, 2, 16, 64), None)
    with pytest.raises(ValueError):
        tree.tree_commit(i32(1, 4), i32(1, 4), i32(1, 4), i32(1), i32(1), i32(1, 2), bf(2, 1, 3, 2, 16, 64))


# ---- the operators together -----------------------------------------------------------------
def test_tree_decoding_emits_what_autoregressive_decoding_would():
    """The example's model: every token that tree decoding emits is, within
    2^-4 of the logits (bf16 cache and attention; logits of about +-10), the one
    that a pass over the emitted sequence itself, as a chain, has largest, and
    trees need fewer passes than tokens."""
    import os
    import sys
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import tree_decode as E
    from paper_2504_18583_gb300 import tree
    model = E.Model()
    g = torch.Generator().manual_seed(5)
    prompts = [torch.randint(0, model.vocab, (n,), generator=g).tolist() for n in (40, 7, 100)]
    n_new = 64
    out, passes = E.generate(model, prompts, n_new)
    assert passes < n_new
    B, pages = len(out), 16
    table = torch.arange(B * pages, dtype=torch.int32, device="cuda").view(B, pages)
    pool = torch.zeros((model.layers, 2, B * pages, model.Hkv, PAGE, model.hd), dtype=torch.bfloat16, device="cuda")
    N = max(len(o) for o in out)
    assert [len(o) - len(p) for o, p in zip(out, prompts)] == [n_new] * B
    chain, nodes, ctx = dev([[i - 1 for i in range(N)]] * B), dev([len(o) for o in out]), dev([0] * B)
    tokens = dev([o + [0] * (N - len(o)) for o in out])
    plan = tree.tree_plan(chain, nodes, ctx, table, B * pages)
    logits = model.forward(tokens, plan, pool, table, ctx, nodes).cpu()
    for b, (o, p) in enumerate(zip(out, prompts)):
        for i in range(len(p) - 1, len(o) - 1):
            assert logits[b, i, o[i + 1]] >= logits[b, i].max() - 2.0 ** -4, (b, i)


def test_calls_in_a_cuda_graph(tree):
    """The whole step captured once and replayed on other inputs."""
    rs = np.random.RandomState(3)
    B, N, Hq, Hkv, hd, n_pages = 3, 9, 8, 2, 64, 40
    g = torch.Generator(device="cuda").manual_seed(6)
    pool = torch.randn((1, 2, n_pages, Hkv, PAGE, hd), generator=g, device="cuda").bfloat16()
    lens, nodes = dev([100, 30, 7]), dev([9, 4, 6])
    table = dev(np.arange(36).reshape(3, 12))
    parents = dev([random_tree(rs, N) for _ in range(B)])
    qkv = torch.randn((B * N, (Hq + 2 * Hkv) * hd), generator=g, device="cuda").bfloat16()
    logits, u = torch.randn((B * N, 500), generator=g, device="cuda"), torch.rand(B * N, generator=g, device="cuda")
    tokens = dev(rs.randint(0, 500, (B, N)))
    freq, _ = tree.rope_frequencies(hd)

    def step():
        mask, pos, slots = tree.tree_plan(parents, nodes, lens, table, n_pages)
        q = tree.qk_norm_rope(qkv, Hq, Hkv, pos.view(-1), slots.view(-1), pool[0, 0], pool[0, 1], freq)
        o = tree.tree_attention(q.view(B, N, Hq, hd), pool[0, 0], pool[0, 1], table, lens, nodes, mask)
        token, logp = tree.sample(logits, u)
        return (o, token, logp) + tuple(tree.tree_commit(token.view(B, N), tokens, parents, nodes, lens, table, pool))

    kept = pool.clone()
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    pool.copy_(kept)
    with torch.cuda.graph(graph):
        outs = step()
    for seed in range(3):
        g.manual_seed(100 + seed)
        qkv.copy_(torch.randn(qkv.shape, generator=g, device="cuda"))
        logits.copy_(torch.randn(logits.shape, generator=g, device="cuda"))
        u.copy_(torch.rand(u.shape, generator=g, device="cuda"))
        pool.copy_(kept)
        want = [x.clone() for x in step()] + [pool.clone()]
        pool.copy_(kept)
        graph.replay()
        for x, y in zip(want, list(outs) + [pool]):
            assert torch.equal(x, y)
