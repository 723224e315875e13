"""The operators of a serving loop against plain 64-bit implementations.

Tolerances, with u the output type's unit roundoff (2^-8 bf16, 2^-11 fp16):
chunk attention, as tree attention, rounds probabilities and the output:
u |o| + 2 u sum_j w_j |v_j|, the second u covering the scores' 32-bit products
(relative error of a weight below 2^-12 at the scores used); in fp16 weights
below 2^-21 of the largest are multiples of 2^-32 of it, which adds 2^-32 sum |v|.
An 8-bit cache's entries are read as fp16: held to +-65504 and rounded to multiples
of 2^-24, which changes none of most tests' entries (codes are multiples of 2^-9 up
to 448, their powers of two between 2^-15 and 2^7).  Probabilities are then fp16 too,
so that the bf16 tolerance has room to spare.

Codes of the 8-bit cache are off by half a step of e4m3 at most: 2^-4 of the entry
or 2^-10 of the row's scale, plus 2^-18 of the head's largest entry for the 32-bit
norm and rotation before it (as in the 16-bit write's test); a row's exponent is
the definition's unless its largest entry lies within 2^-18 of a border.

Adjusted logits are rounded once, u |y|, after at most five 32-bit operations on
values no larger than |z| (r + 1 / r) + f c + p + sum |bias|, each off by 2^-24 of
that: 2^-21 of it in all, and 2^-24 more of it for each further bias of a token."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

ROUND = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
BF, FP = torch.bfloat16, torch.float16
PAGE = 16


@pytest.fixture(scope="module")
def tree():
    from paper_2504_18583_gb300 import _build, tree
    _build.build()
    return tree


def dev(a, dtype=torch.int32):
    return torch.tensor(np.asarray(a), dtype=dtype, device="cuda")


# ---- chunk attention --------------------------------------------------------------
def quantise(x):
    """Codes and biased exponents of rows, by the definition, in 64 bits."""
    most = x.double().abs().amax(-1)
    e = torch.ceil(torch.log2(torch.clamp(most, min=1e-300) / 448)).clamp(-126, 127)
    e = torch.where(most > 448 * torch.exp2(e), e + 1, e)
    codes = (x.double() * torch.exp2(-e)[..., None]).float().to(torch.float8_e4m3fn)
    return codes, (e + 127).to(torch.uint8)


class Case:
    """A batch of chunks over a pool of shuffled pages; what lies outside the sequences is NaN."""

    def __init__(self, dtype, Hq, Hkv, hd, new, ctx, eight=False, seed=0, extra_rows=0, table_pages=None, spread=1.5):
        rs, g = np.random.RandomState(seed), torch.Generator(device="cuda").manual_seed(seed)
        self.dtype, self.Hq, self.Hkv, self.hd, self.new, self.ctx, self.eight = dtype, Hq, Hkv, hd, new, ctx, eight
        B = len(new)
        need = [-(-(c + n) // PAGE) for c, n in zip(ctx, new)]
        self.n_pages = sum(need) + 2
        order = rs.permutation(self.n_pages)
        P = table_pages or max(max(need), 1) + 1
        self.table = np.full((B, P), 10 ** 6)
        at = 0
        for b, n in enumerate(need):
            self.table[b, :min(n, P)] = order[at:at + n][:P]
            at += n
        self.starts = np.cumsum([0] + list(new))
        self.T = int(self.starts[-1]) + extra_rows
        self.q = (spread * torch.randn((self.T, Hq, hd), generator=g, device="cuda")).to(dtype)
        k = torch.randn((self.n_pages, Hkv, PAGE, hd), generator=g, device="cuda")
        v = torch.randn((self.n_pages, Hkv, PAGE, hd), generator=g, device="cuda")
        live = torch.zeros((self.n_pages, PAGE), dtype=torch.bool, device="cuda")
        for b in range(B):
            for i in range(min(need[b], P)):
                live[self.table[b, i], :max(0, min(PAGE, ctx[b] + new[b] - i * PAGE))] = True
        dead = ~live[:, None, :, None]
        if eight:
            size = torch.exp(torch.randn((2, self.n_pages, Hkv, PAGE, 1), generator=g, device="cuda"))
            (self.k, self.ks), (self.v, self.vs) = quantise(k * size[0].clamp(0.2, 1.5)), quantise(v * size[1])
            for x, s in ((self.k, self.ks), (self.v, self.vs)):
                x.view(torch.uint8).masked_fill_(dead, 0x7F)
                s.masked_fill_(dead[..., 0], 0xFF)
        else:
            self.k, self.v = (x.masked_fill(dead, float("nan")).to(dtype) for x in (k, v))
            self.ks = self.vs = None

    def values(self, which, pages):
        x = getattr(self, which)[torch.as_tensor(pages, device="cuda").long()] if not self.eight else \
            getattr(self, which).view(torch.uint8)[torch.as_tensor(pages, device="cuda").long()].view(torch.float8_e4m3fn)
        x = x.double()
        if self.eight:
            e = getattr(self, which + "s")[torch.as_tensor(pages, device="cuda").long()].double() - 127
            x = x * torch.where(e < 128, torch.exp2(e), float("nan"))[..., None]
            x = x.clamp(-65504, 65504).half().double()
        return x.transpose(0, 1).reshape(self.Hkv, -1, self.hd)

    def call(self, tree, window=0, sinks=0, scale=None, **kw):
        return tree.chunk_attention(self.q, self.k, self.v, dev(self.table), dev(self.starts), dev(self.ctx), scale=scale,
                                    window=window, sinks=sinks, k_scale=self.ks, v_scale=self.vs, **kw)

    def sees(self, b, n_keys, window, sinks):
        pos = torch.arange(self.ctx[b], self.ctx[b] + self.new[b], device="cuda")[:, None]
        j = torch.arange(n_keys, device="cuda")[None]
        sees = j <= pos
        if window:
            sees &= (pos - j < window) | (j < sinks)
        return sees

    def reference(self, window=0, sinks=0, scale=None):
        """Outputs and their tolerances in 64 bits; rows that see nothing are 0."""
        scale = self.hd ** -0.5 if scale is None else scale
        u, group = ROUND[self.dtype], self.Hq // self.Hkv
        out = torch.full((self.T, self.Hq, self.hd), float("nan"), dtype=torch.float64, device="cuda")
        tol = torch.zeros_like(out)
        for b, n in enumerate(self.new):
            if n == 0:
                continue
            pages = [int(p) if 0 <= p < self.n_pages else -1 for p in self.table[b, :-(-(self.ctx[b] + n) // PAGE)]]
            K, V = (self.values(w, [max(p, 0) for p in pages]) for w in "kv")
            here = torch.tensor([p >= 0 for p in pages], device="cuda").repeat_interleave(PAGE)
            sees = self.sees(b, len(here), window, sinks) & here
            for h in range(self.Hq):
                rows = slice(int(self.starts[b]), int(self.starts[b]) + n)
                z = (self.q[rows, h].double() @ torch.nan_to_num(K[h // group]).T) * scale
                bad = sees & torch.isnan(K[h // group]).any(-1)
                z = torch.where(bad, float("nan"), z).masked_fill(~sees, float("-inf"))
                w = torch.softmax(z, -1)
                w = torch.where(sees.any(-1, keepdim=True), w, 0.0)
                v = V[h // group]
                clean = torch.nan_to_num(v, nan=0.0, posinf=0.0, neginf=0.0)
                o = w @ clean
                odd = torch.where(torch.isnan(v) | torch.isinf(v), v, 0.0)
                if not torch.isfinite(v).all():
                    for j in torch.nonzero(~torch.isfinite(v).all(-1))[:, 0].tolist():
                        o = torch.where(sees[:, j, None], o + odd[j], o)
                out[rows, h] = o
                mag = torch.nan_to_num(w) @ clean.abs()
                tol[rows, h] = u * o.abs() + 2 * u * mag
                if self.dtype == FP:
                    tol[rows, h] += 2.0 ** -32 * clean.abs().sum(0).amax() + 2.0 ** -24
        return out, tol

    def check(self, tree, window=0, sinks=0, scale=None, **kw):
        want, tol = self.reference(window, sinks, scale)
        live = int(self.starts[-1])
        out = torch.full((self.T, self.Hq, self.hd), 7.25, dtype=self.dtype, device="cuda")
        got = self.call(tree, window, sinks, scale, out=out, **kw)
        assert got.data_ptr() == out.data_ptr()
        assert (got[live:] == 7.25).all()  # rows of no sequence are left as they were
        got, want, tol = got[:live].double(), want[:live], tol[:live]
        assert torch.equal(torch.isnan(got), torch.isnan(want))
        inf = torch.isinf(want)
        assert torch.equal(got[inf], want[inf])
        fine = torch.isfinite(want)
        err = (got - want).abs()[fine]
        assert (err <= tol[fine]).all(), float((err / tol[fine]).max())


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("Hq,Hkv,hd,new,ctx", [
    (8, 2, 128, [1], [0]),                                # one key
    (8, 2, 64, [1, 1, 1], [15, 16, 127]),                 # ends of pages and tiles
    (32, 8, 128, [1], [700]),
    (8, 2, 64, [5, 0, 33], [60, 9, 0]),                   # a sequence without new tokens
    (4, 4, 128, [130, 7], [3, 200]),                      # a head each: 130 rows are two blocks of one group
    (6, 2, 64, [100, 61], [10, 64]),                      # three query heads a key/value head
    (14, 2, 128, [40, 19], [100, 0]),                     # seven: blocks begin inside a token
    (64, 1, 64, [9], [130]),
    (16, 4, 128, [300], [77]),
    (16, 4, 64, [257, 1, 1], [0, 3000, 511]),
])
def test_chunks(tree, eight, dtype, Hq, Hkv, hd, new, ctx):
    Case(dtype, Hq, Hkv, hd, new, ctx, eight, seed=hd + len(new)).check(tree)


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (5, 0), (64, 4), (128, 0), (129, 33), (200, 128), (300, 200), (4000, 4),
                                          (100, 5000), (2 ** 31 - 1, 0), (100, 2 ** 31 - 1)])
def test_windows_and_first_tokens(tree, eight, window, sinks):
    Case(BF, 8, 2, 64, [1, 150, 3], [900, 500, 40], eight, seed=window % 1000 + sinks % 1000).check(tree, window, sinks)
    Case(FP, 4, 2, 128, [1, 1, 1], [1000, 127, 0], eight, seed=window % 1000 + 1).check(tree, window, sinks)


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("dtype", [BF, FP])
def test_tiles_that_are_not_loaded_whole(tree, dtype, hd, eight):
    """Behind what a tile needs of its pages lies what shared memory held before: NaN of another call's caches."""
    before = Case(dtype, 32, 8, hd, [1] * 40, [2000] * 40, eight)
    for x in (before.k, before.v):
        x.view(torch.uint8).fill_(0x7F) if eight else x.fill_(float("nan"))
    for new, ctx, window, sinks in (([1], [1023], 1, 1), ([1], [1000], 200, 112), ([40], [1007], 1, 64), ([150], [3000], 800, 200),
                                    ([1, 1, 300], [111, 4095, 2047], 700, 17), ([5], [64], 0, 0)):
        before.call(tree)
        Case(dtype, 4, 2, hd, new, ctx, eight, seed=len(new)).check(tree, window, sinks)


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("dtype,Hq,Hkv,hd,new,ctx", [
    (BF, 32, 8, 128, [1], [20000]),                       # parts of units, many to join
    (BF, 4, 1, 64, [1, 1], [30000, 100]),
    (FP, 8, 2, 128, [64], [6000]),                        # one block a unit, more CTAs than units
    (BF, 8, 8, 64, [700], [1500]),                        # ranges that begin inside a unit
    (FP, 32, 8, 128, [513, 1, 1, 129], [2000, 5000, 31, 0]),
    (BF, 64, 8, 128, [256], [4000]),
])
def test_units_in_parts(tree, eight, dtype, Hq, Hkv, hd, new, ctx):
    Case(dtype, Hq, Hkv, hd, new, ctx, eight, seed=new[0]).check(tree)


@pytest.mark.parametrize("batch,new", [(64, 1), (65, 1), (130, 2), (600, 1), (70, 40)])
def test_many_sequences(tree, batch, new):
    """More sequences than a CTA keeps at hand, or than it has threads; some without new tokens."""
    rs = np.random.RandomState(batch)
    n = [int(x) for x in np.where(rs.rand(batch) < 0.2, 0, rs.randint(1, new + 1, batch))]
    Case(BF, 4, 2, 64, n, [int(x) for x in rs.randint(0, 400, batch)], batch % 2 == 0, seed=batch).check(tree)


def test_nothing_to_do(tree):
    Case(BF, 4, 2, 64, [0, 0, 0], [5, 100, 0], extra_rows=3).check(tree)
    c = Case(BF, 4, 2, 64, [3], [5])
    assert tree.chunk_attention(c.q[:0], c.k, c.v, dev(c.table), dev([0, 0]), dev([5])).shape == (0, 4, 64)


@pytest.mark.parametrize("eight", [False, True])
def test_rows_of_no_sequence_are_left(tree, eight):
    Case(BF, 8, 2, 128, [70, 1], [30, 200], eight, extra_rows=200).check(tree)
    c = Case(BF, 8, 2, 128, [70, 3], [30, 200], eight)
    c.T, c.q = 71, c.q[:71].contiguous()  # starts that pass the rows given: those outside do not exist
    want, tol = Case.reference(_cut(c, 1), 0, 0)
    got = c.call(tree)
    assert ((got.double() - want).abs() <= tol).all()


def _cut(c, left):
    """The same batch with `left` rows of its last sequence."""
    import copy
    d = copy.copy(c)
    d.new = list(c.new[:-1]) + [left]
    d.starts = np.cumsum([0] + d.new)
    return d


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("hd", [64, 128])
def test_pages_outside_the_pool_and_past_the_table(tree, hd, eight):
    c = Case(BF, 8, 2, hd, [40, 1, 1], [300, 250, 20], eight, seed=3)
    c.table[0, 2] = -1
    c.table[0, 9] = c.n_pages
    c.table[1, 0:8] = 2 ** 31 - 1  # a whole tile
    c.table[2, :2] = -5            # nothing left to see
    c.check(tree)
    c.check(tree, window=64)
    Case(BF, 8, 2, hd, [60, 1], [100, 300], eight, table_pages=9).check(tree)
    Case(BF, 8, 2, hd, [60, 1], [100, 3000], eight, table_pages=9).check(tree, window=50, sinks=3)


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("new,ctx,window,sinks", [([100, 1], [200, 90], 0, 0), ([150], [300], 60, 5), ([20], [1200], 500, 0),
                                                  ([300, 2], [9000, 4], 0, 0)])
def test_infinities_and_nan_reach_only_rows_that_see_them(tree, eight, dtype, new, ctx, window, sinks):
    c = Case(dtype, 8, 2, 64, new, ctx, eight, seed=11)
    rs = np.random.RandomState(5)

    def put(which, pos, kind):
        page, head = int(c.table[0, pos // PAGE]), int(rs.randint(2))
        if eight and which == "v" and kind == "scale":
            c.vs[page, head, pos % PAGE] = 255
        elif eight:
            getattr(c, which).view(torch.uint8)[page, head, pos % PAGE, int(rs.randint(64))] = 0xFF
        else:
            x = float("nan") if which == "k" else (float("inf"), float("-inf"), float("nan"))[rs.randint(3)]
            getattr(c, which)[page, head, pos % PAGE, int(rs.randint(64))] = x

    put("v", ctx[0] + new[0] // 2, "code")
    put("v", ctx[0] + new[0] - 2, "scale")
    put("k", ctx[0] + new[0] // 3, "code")
    if window:
        put("v", ctx[0] + new[0] // 4 - window, "code")
    c.check(tree, window, sinks)


def test_scales(tree):
    for scale in (0.0, -0.3, 1e-3, 2.0):
        Case(BF, 8, 2, 64, [30, 1], [100, 20], seed=2, spread=0.7).check(tree, scale=scale, window=50)


def test_strided_queries_and_caches(tree):
    """Queries as columns of a QKV projection, caches as one layer of a pool with a gap between pages."""
    for eight in (False, True):
        c = Case(FP, 8, 2, 128, [50, 1, 9], [40, 300, 0], eight, seed=8)
        wide = torch.full((c.T, 12 * 128 + 8), float("nan"), dtype=FP, device="cuda")
        wide[:, :1024] = c.q.view(c.T, -1)
        c.q = wide[:, :1024].view(c.T, 8, 128)
        for name in ("k", "v", "ks", "vs"):
            x = getattr(c, name)
            if x is None:
                continue
            y = x.view(torch.uint8) if x.dtype == torch.float8_e4m3fn else x
            apart = torch.zeros((c.n_pages, 3) + tuple(y.shape[1:]), dtype=y.dtype, device="cuda")
            apart[:, 1] = y
            setattr(c, name, apart[:, 1].view(x.dtype))
        c.check(tree, window=100, sinks=2)


def test_offsets_past_32_bits(tree):
    """A cache of more than 2^32 entries of which the last pages are used."""
    for eight in (False, True):
        n_pages, Hkv, hd = 290000, 8, 128
        dt = torch.uint8 if eight else BF
        cache = torch.zeros((2, n_pages, Hkv, PAGE, hd), dtype=dt, device="cuda")
        c = Case(BF, 16, Hkv, hd, [20, 1], [200, 100], eight, seed=4)
        far = n_pages - c.n_pages
        for i, name in enumerate("kv"):
            cache[i, far:] = getattr(c, name).view(dt)
            setattr(c, name, cache[i].view(torch.float8_e4m3fn) if eight else cache[i])
            if eight:
                s = torch.zeros((n_pages, Hkv, PAGE), dtype=torch.uint8, device="cuda")
                s[far:] = getattr(c, name + "s")
                setattr(c, name + "s", s.view(torch.float8_e8m0fnu))
        c.table = np.where(c.table < c.n_pages, c.table + far, 10 ** 7)
        c.n_pages = n_pages
        if eight:
            c.ks, c.vs = c.ks.view(torch.uint8), c.vs.view(torch.uint8)
        c.check(tree)
        del cache, c
        torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("high,low", [(7, -15), (8, -16), (12, -20), (100, -100)])
def test_8_bit_extremes(tree, dtype, high, low):
    """Rows whose powers of two are large and small: held to 65504 and to multiples of 2^-24.  Weights are even, so that
    an output may be as large as the largest entry: it is compared where that is no more than 60000."""
    c = Case(dtype, 8, 2, 64, [30, 1], [200, 150], True, seed=6, spread=0.0)
    c.vs[:, 0][c.vs[:, 0] < 255] = 127 + high
    c.vs[:, 1][c.vs[:, 1] < 255] = 127 + low
    c.ks[c.ks < 255] = 127 - 8
    want, tol = c.reference()
    got = c.call(tree).double()
    fine = want.abs() < 60000
    assert torch.isfinite(got).all() and ((got - want).abs() <= tol)[fine].all()


@pytest.mark.parametrize("hd", [64, 128])
def test_8_bit_cache_with_large_and_small_queries(tree, hd):
    """bf16 queries of any size over an 8-bit cache: rows are scaled to fp16's range and back; the scale keeps scores
    ordinary."""
    for q_size in (2.0 ** 100, 2.0 ** -100, 1e-3, 300.0):
        c = Case(BF, 8, 2, hd, [40, 1], [100, 30], True, seed=7)
        c.ks[c.ks < 255] = 127 - 7
        c.q = (c.q.float() * q_size).to(BF)
        c.q[0] = 0
        c.q[1, :, 1:] = 0
        c.check(tree, scale=0.05 / q_size)


def test_one_workspace_for_all_sizes_and_repeatable(tree):
    sizes = [([1], [5000]), ([300, 1], [1000, 0]), ([1] * 9, [400] * 9), ([64], [3000])]
    ws = tree.chunk_attention_workspace(400, 1, 32, 8, 128)
    for new, ctx in sizes * 2:
        c = Case(BF, 16, 4, 128, new, ctx, seed=sum(new))
        c.check(tree, workspace=ws)
        assert torch.equal(c.call(tree, workspace=ws), c.call(tree))
    assert int(ws[:1296].sum()) == 0


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("new,ctx", [([1], [3000]), ([300, 2], [10, 700]), ([1] * 70, [30] * 70)])
def test_after_a_wait_ran_out(tree, new, ctx, eight):
    """The mark that a wait leaves when it runs out, set by hand: NaN until the workspace is zeroed again."""
    c = Case(BF, 8, 2, 64, new, ctx, eight, extra_rows=2)
    ws = tree.chunk_attention_workspace(c.T, len(new), 8, 2, 64)
    want = c.call(tree, workspace=ws)[:-2]
    ws.view(torch.int32)[320] = 1
    for _ in range(2):
        out = torch.full_like(c.q, 3.0)
        assert torch.isnan(c.call(tree, workspace=ws, out=out)[:-2]).all() and (out[-2:] == 3.0).all()
    ws[:4096].zero_()
    assert torch.equal(c.call(tree, workspace=ws)[:-2], want)


def test_graphs_and_streams(tree):
    """Captured calls (their first in the process on that stream among them) replayed with other lengths, beside eager
    calls on another stream."""
    c = Case(BF, 8, 2, 128, [40, 1], [300, 900], seed=9)
    table, starts, ctx = dev(c.table), dev(c.starts), dev(c.ctx)
    call = lambda: tree.chunk_attention(c.q, c.k, c.v, table, starts, ctx, window=128, sinks=4)  # noqa: E731
    want = call()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        assert torch.equal(call(), want)
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        first, second = call(), call()
    for _ in range(3):
        first.zero_()
        second.zero_()
        graph.replay()
        with torch.cuda.stream(s):
            beside = call()
        torch.cuda.synchronize()
        assert torch.equal(first, want) and torch.equal(second, want) and torch.equal(beside, want)
    starts.copy_(dev([0, 7, 8]))
    ctx.copy_(dev([333, 20]))
    graph.replay()
    assert torch.equal(first[:8], call()[:8])


def test_chunk_refusals(tree):
    c = Case(BF, 8, 2, 64, [5, 1], [20, 3])
    t, s, x = dev(c.table), dev(c.starts), dev(c.ctx)
    ok = dict(q=c.q, k_cache=c.k, v_cache=c.v, page_table=t, starts=s, ctx_len=x)
    eight = tree.quantized_cache(c.n_pages, 2, 64)
    for edit in (dict(q=c.q.float()), dict(q=c.q.cpu()), dict(q=c.q[:, :, ::2]), dict(k_cache=c.k.half()), dict(v_cache=c.v[:-1]),
                 dict(starts=s[:-1]), dict(starts=s.long()), dict(ctx_len=x[:1]), dict(page_table=t.long()),
                 dict(out=torch.empty_like(c.q).float()), dict(k_scale=eight[2]), dict(k_scale=eight[2], v_scale=eight[3]),
                 dict(k_cache=eight[0], v_cache=eight[1]), dict(workspace=torch.zeros(4096)),
                 dict(k_cache=eight[0], v_cache=eight[1], k_scale=eight[2][:1], v_scale=eight[3])):
        with pytest.raises(ValueError):
            tree.chunk_attention(**{**ok, **edit})
    from paper_2504_18583_gb300.pard import PardError
    for edit in (dict(window=-1), dict(sinks=-1), dict(scale=float("nan")), dict(q=c.q[:, :7]),
                 dict(workspace=torch.zeros(4096, device="cuda", dtype=torch.uint8))):
        with pytest.raises((PardError, ValueError)):
            tree.chunk_attention(**{**ok, **edit})


# ---- the 8-bit cache's write --------------------------------------------------------
def rotate64(x, gain, eps, pos, freq, rot, interleaved, amp):
    y = x.double()
    if gain is not None:
        y = y / (y.square().mean(-1, keepdim=True) + eps).sqrt() * gain.double()
    ang = (pos.double()[:, None] * freq.double()[None])[:, None]
    c, s = amp * ang.cos(), amp * ang.sin()
    out = y.clone()
    ia, ib = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    out[..., ia], out[..., ib] = y[..., ia] * c - y[..., ib] * s, y[..., ia] * s + y[..., ib] * c
    return out


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("T,Hq,Hkv,hd,rot,interleaved,norm", [
    (1, 32, 8, 128, 128, False, True), (9, 8, 2, 64, 64, True, True), (37, 6, 3, 64, 32, False, False),
    (400, 8, 2, 128, 64, True, True), (1001, 32, 8, 64, 64, False, True), (5, 4, 1, 128, 0, False, True), (33, 7, 7, 64, 16, False, False),
])
def test_quantized_write(tree, dtype, T, Hq, Hkv, hd, rot, interleaved, norm):
    g = torch.Generator(device="cuda").manual_seed(T)
    rs = np.random.RandomState(T)
    n_pages = -(-T // PAGE) + 3
    size = torch.exp(torch.randn((T, Hq + 2 * Hkv, 1), generator=g, device="cuda") * 2)
    x = torch.randn((T, Hq + 2 * Hkv, hd), generator=g, device="cuda") * size
    x[0, -1] = 0.0  # a row of zeros
    x = x.to(dtype)
    wide = torch.zeros((T, (Hq + 2 * Hkv) * hd + 16), dtype=dtype, device="cuda")
    wide[:, :-16] = x.view(T, -1)
    gains = [(1 + 0.3 * torch.randn(hd, generator=g, device="cuda")).to(dtype) if norm else None for _ in range(2)]
    pos = dev(rs.randint(0, 200000, T))
    slots = rs.permutation(n_pages * PAGE)[:T]
    slots[T // 2] = -1 if T > 1 else slots[0]
    if T > 4:
        slots[1] = n_pages * PAGE
    freq = torch.tensor(1e4 ** (-2.0 * np.arange(rot // 2) / max(rot, 1)), dtype=torch.float32, device="cuda") if rot else None
    k, v, ks, vs = tree.quantized_cache(n_pages, Hkv, hd)
    for c in (k, v):
        c.view(torch.uint8).fill_(0x55)
    for s in (ks, vs):
        s.view(torch.uint8).fill_(99)
    q = tree.qk_norm_rope(wide[:, :-16], Hq, Hkv, pos, dev(slots, torch.int64), k, v, freq, q_gain=gains[0], k_gain=gains[1], eps=1e-5,
                          interleaved=interleaved, amplitude=1.25, k_scale=ks, v_scale=vs)
    kc, vc = (torch.zeros((n_pages, Hkv, PAGE, hd), dtype=dtype, device="cuda") for _ in range(2))
    same = tree.qk_norm_rope(wide[:, :-16], Hq, Hkv, pos, dev(slots, torch.int64), kc, vc, freq, q_gain=gains[0], k_gain=gains[1],
                             eps=1e-5, interleaved=interleaved, amplitude=1.25)
    assert torch.equal(q, same)
    want = {"k": x[:, Hq:Hq + Hkv].double(), "v": x[:, Hq + Hkv:].double()}
    if rot:
        want["k"] = rotate64(x[:, Hq:Hq + Hkv], gains[1], 1e-5, pos, freq, rot, interleaved, 1.25)
    elif norm:
        y = x[:, Hq:Hq + Hkv].double()
        want["k"] = y / (y.square().mean(-1, keepdim=True) + 1e-5).sqrt() * gains[1].double()
    written = torch.zeros((n_pages, PAGE), dtype=torch.bool, device="cuda")
    for t in range(T):
        if 0 <= slots[t] < n_pages * PAGE:
            written[slots[t] // PAGE, slots[t] % PAGE] = True
    live = torch.tensor([0 <= s < n_pages * PAGE for s in slots], device="cuda")
    at = torch.tensor(np.clip(slots, 0, n_pages * PAGE - 1), device="cuda")
    for name, codes, scale in (("k", k, ks), ("v", v, vs)):
        untouched = ~written[:, None, :].expand(-1, Hkv, -1)
        assert (codes.view(torch.uint8)[untouched] == 0x55).all() and (scale.view(torch.uint8)[untouched] == 99).all()
        y = want[name][live]
        e = scale.view(torch.uint8)[at // PAGE, :, at % PAGE][live].double() - 127
        got = codes.view(torch.uint8)[at // PAGE, :, at % PAGE][live].view(torch.float8_e4m3fn).double() * torch.exp2(e)[..., None]
        most = y.abs().amax(-1)
        slack = 2.0 ** -18 if name == "k" else 0.0
        assert (most * (1 - slack) <= 448 * torch.exp2(e)).all()
        assert ((most * (1 + slack) > 224 * torch.exp2(e)) | (e == -126)).all()
        tol = torch.maximum(2.0 ** -4 * y.abs(), 2.0 ** -10 * torch.exp2(e)[..., None]) + slack * most[..., None]
        assert ((got - y).abs() <= tol).all()


def test_quantized_write_not_finite(tree):
    """Infinities and NaN become NaN, count for no exponent, and touch no other entry; exponents at 448's borders."""
    hd, T = 64, 6
    x = torch.ones((T, 3, hd))
    x[0, 1:, 3] = float("inf")
    x[1, 1:, 5], x[1, 1:, 6] = float("nan"), float("-inf")
    x[2] = float("nan")
    x[3, 1:, 0] = 448.0
    x[4, 1:, 0] = 450.0
    x[5] = 2.0 ** -133
    x = x.to(BF)
    k, v, ks, vs = tree.quantized_cache(2, 1, hd)
    tree.qk_norm_rope(x.view(T, -1).cuda(), 1, 1, dev(range(T)), dev(range(T), torch.int64), k, v, None, k_scale=ks, v_scale=vs)
    for codes, scale in ((k, ks), (v, vs)):
        e = scale.view(torch.uint8)[0, 0, :T].cpu().int()
        got = codes.view(torch.uint8)[0, 0, :T].cpu().view(torch.float8_e4m3fn).double() * torch.exp2(e.double() - 127)[:, None]
        assert e.tolist() == [119, 119, 1, 127, 128, 1]
        want = torch.where(torch.isfinite(x[:, 1]), x[:, 1].double(), float("nan"))
        want[4, 0] = 448.0  # 225 lies between 224 and 240
        # 2^-133 is 2^-7 * 2^-126, four of e4m3's smallest steps: exact at the lowest exponent
        assert torch.equal(torch.isnan(got), torch.isnan(want))
        fine = ~torch.isnan(want)
        assert torch.equal(got[fine], want[fine])


def test_quantized_write_refusals(tree):
    k, v, ks, vs = tree.quantized_cache(4, 2, 64)
    x = torch.zeros((3, 8 * 64), dtype=BF, device="cuda")
    args = lambda **kw: {**dict(qkv=x, n_q_heads=4, n_kv_heads=2, pos=dev([0, 1, 2]), slots=dev([0, 1, 2], torch.int64), k_cache=k,  # noqa: E731
                                v_cache=v, inv_freq=None, k_scale=ks, v_scale=vs), **kw}
    tree.qk_norm_rope(**args())
    tree.qk_norm_rope(**args(k_scale=ks.view(torch.uint8), v_scale=vs.view(torch.uint8)))
    for edit in (dict(k_scale=None), dict(v_scale=None), dict(k_scale=None, v_scale=None), dict(k_cache=k.view(torch.uint8)),
                 dict(k_scale=ks[:2]), dict(k_scale=ks.float()), dict(k_scale=ks[:, :, ::2]), dict(n_kv_heads=1, n_q_heads=6)):
        with pytest.raises(ValueError):
            tree.qk_norm_rope(**args(**edit))


# ---- adjusted logits ------------------------------------------------------------------
def adjust64(z, N, hist=None, hist_len=None, prompt_len=None, rep=None, freq=None, pres=None, ids=None, bias=None, allowed=None,
             tokens=None, mask=None):
    """Values and tolerances in 64 bits, row by row."""
    dtype, y = z.dtype, z.double().cpu().numpy().copy()
    R, V = y.shape
    tol = np.zeros_like(y)
    for r in range(R):
        b, i = divmod(r, N)
        said, prompt = [], []
        if hist is not None:
            n = min(max(int(hist_len[b]), 0), hist.shape[1])
            p = min(max(int(prompt_len[b]), 0), n) if prompt_len is not None else 0
            prompt, said = hist[b, :p].tolist(), hist[b, p:n].tolist()
        if tokens is not None:
            said = said + [int(tokens[b, j]) for j in range(N) if int(mask[b, i, j // 64]) >> (j % 64) & 1]
        count, size = {}, np.abs(y[r])
        for t in said:
            count[t] = count.get(t, 0) + 1
        r_, f_, p_ = (float(x[b]) if x is not None else d for x, d in ((rep, 1.0), (freq, 0.0), (pres, 0.0)))
        for t in set(said) | set(prompt):
            if 0 <= t < V:
                y[r, t] = y[r, t] / r_ if y[r, t] > 0 else y[r, t] * r_
                size[t] = size[t] * (r_ + 1 / r_) + abs(f_) * count.get(t, 0) + abs(p_)
        for t, c in count.items():
            if 0 <= t < V:
                y[r, t] = y[r, t] - f_ * c - p_
        many = np.zeros(V)
        if ids is not None:
            for t, x in zip(ids[b].tolist(), bias[b].tolist()):
                if 0 <= t < V:
                    y[r, t] += x
                    size[t] += abs(x)
                    many[t] += 1
        with np.errstate(invalid="ignore"):
            tol[r] = ROUND[dtype] * np.abs(y[r]) + (2.0 ** -21 + many * 2.0 ** -24) * size
        if allowed is not None:
            w = np.ascontiguousarray(allowed[r]).view(np.uint8)
            y[r, np.unpackbits(w, bitorder="little")[:V] == 0] = -np.inf
    return y, tol


def check_adjust(tree, z, N=1, out=None, **kw):
    names = dict(hist="history", hist_len="hist_len", prompt_len="prompt_len", rep="repetition", freq="frequency", pres="presence",
                 ids="bias_ids", bias="bias", allowed="allowed", tokens="tokens", mask="mask")
    types = dict(rep=torch.float32, freq=torch.float32, pres=torch.float32, bias=torch.float32, mask=torch.int64)
    for n in ("rep", "freq", "pres", "bias"):
        if kw.get(n) is not None:
            kw[n] = np.asarray(kw[n], np.float32)
    want, tol = adjust64(z, N, **kw)
    given = {names[n]: dev(a.view(np.int64) if n == "mask" else a.view(np.int32) if n == "allowed" else a, types.get(n, torch.int32))
             for n, a in kw.items() if a is not None}
    before = z.clone()
    got = tree.adjust_logits(z, out=out, **given)
    if out is not z:
        assert torch.equal(z.view(torch.uint8) if z.is_contiguous() else z.nan_to_num(), before.view(torch.uint8) if z.is_contiguous() else before.nan_to_num())
    g = got.double().cpu().numpy()
    assert np.array_equal(np.isnan(g), np.isnan(want))
    inf = np.isinf(want)
    assert np.array_equal(g[inf], want[inf])
    fine = np.isfinite(want)
    over = np.abs(want[fine]) > float(torch.finfo(z.dtype).max) * (1 - 2.0 ** -9)
    err = np.abs(g[fine] - want[fine])[~over]
    assert (err <= tol[fine][~over]).all(), (err - tol[fine][~over]).max()
    return got


def words_of(bits):
    R, V = bits.shape
    W = -(-V // 32)
    full = np.zeros((R, W * 32), np.uint8)
    full[:, :V] = bits
    return np.packbits(full, axis=1, bitorder="little").view(np.uint32)


def tree_mask(rs, B, N):
    words = np.zeros((B, N, -(-N // 64)), np.uint64)
    for b in range(B):
        for i in range(N):
            if i:
                words[b, i] = words[b, rs.randint(max(0, i - 5), i)]
            words[b, i, i // 64] |= np.uint64(1) << np.uint64(i % 64)
    return words


@pytest.mark.parametrize("dtype", [torch.float32, BF, FP])
@pytest.mark.parametrize("B,N,V,L,M,grammar,branch", [
    (1, 1, 1, 3, 0, False, False), (1, 1, 7, 0, 2, True, False), (2, 1, 1000, 50, 5, True, False), (3, 5, 1031, 200, 9, True, True),
    (1, 29, 4099, 300, 20, False, True), (2, 70, 2048, 100, 0, True, True), (2, 256, 333, 40, 3, True, True), (5, 3, 5000, 1000, 300, True, False),
    (70, 1, 9001, 64, 1, False, False), (1, 2, 262144, 5000, 2047, True, False), (2, 600, 100, 10, 0, False, False),
])
def test_adjust(tree, dtype, B, N, V, L, M, grammar, branch):
    rs = np.random.RandomState(V + N)
    g = torch.Generator(device="cuda").manual_seed(V)
    z = (4 * torch.randn((B * N, V), generator=g, device="cuda")).to(dtype)
    few = rs.randint(-2, V + 2, max(4, V // 20))  # ids that come back, some outside
    kw = dict(hist=few[rs.randint(0, len(few), (B, L))] if L else None, hist_len=rs.randint(-1, L + 3, B) if L else None,
              prompt_len=rs.randint(-1, L + 3, B) if L else None, rep=rs.uniform(0.7, 1.5, B), freq=rs.uniform(-0.5, 0.5, B),
              pres=rs.uniform(-1, 1, B), ids=few[rs.randint(0, len(few), (B, M))] if M else None,
              bias=rs.uniform(-5, 5, (B, M)) if M else None, allowed=words_of(rs.rand(B * N, V) < 0.4) if grammar else None)
    if branch:
        kw.update(tokens=few[rs.randint(0, len(few), (B, N))], mask=tree_mask(rs, B, N))
    check_adjust(tree, z, N, **kw)


def test_adjust_one_thing_at_a_time(tree):
    rs = np.random.RandomState(1)
    z = torch.randn((6, 515), generator=torch.Generator().manual_seed(3)).cuda()
    hist = rs.randint(0, 515, (3, 40))
    common = dict(hist=hist, hist_len=[40, 7, 0])
    for kw in (dict(rep=[1.3, 0.5, 2.0]), dict(freq=[0.25, -1.0, 3.0]), dict(pres=[1.0, 2.0, -3.0]), dict(rep=[1.3, 1, 1], prompt_len=[20, 100, 3])):
        check_adjust(tree, z, 2, **{k: np.asarray(v) for k, v in {**common, **kw}.items()})
    check_adjust(tree, z, 2, ids=np.array([[3, 3, 514, -1], [515, 0, 0, 0], [2 ** 31 - 1, -2 ** 31, 9, 3]]), bias=rs.uniform(-9, 9, (3, 4)))
    check_adjust(tree, z, 1, allowed=words_of(rs.rand(6, 515) < 0.5))
    got = check_adjust(tree, z, 1, allowed=np.zeros((6, 17), np.uint32))  # nothing allowed
    assert (got == float("-inf")).all()
    assert (tree.sample(got, torch.zeros(6, device="cuda"))[0] == -1).all()
    assert torch.equal(tree.adjust_logits(z), z)


@pytest.mark.parametrize("dtype", [torch.float32, BF, FP])
def test_adjust_odd_values_and_rows_apart(tree, dtype):
    rs = np.random.RandomState(2)
    wide = torch.randn((4, 1201), generator=torch.Generator().manual_seed(3)).to(dtype).cuda()
    wide[0, 5], wide[0, 6], wide[1, 7], wide[2, 8] = float("nan"), float("inf"), float("-inf"), 0.0
    hist = np.stack([np.arange(0, 40)] * 4)
    kw = dict(hist=hist, hist_len=np.full(4, 40), rep=np.full(4, 1.2), freq=np.full(4, 0.1), pres=np.full(4, 0.2),
              allowed=words_of(rs.rand(4, 1100) < 0.7))
    for first in (0, 1, 8, 33):
        z = wide[:, first:first + 1100]
        check_adjust(tree, z, 1, **kw)
        out = torch.empty((4, 1111), dtype=dtype, device="cuda")[:, 3:1103]
        check_adjust(tree, z, 1, out=out, **kw)
        again = z.clone()
        assert check_adjust(tree, again, 1, out=again, **kw).data_ptr() == again.data_ptr()  # in place
    left = torch.full((4, 1111), 9.0, dtype=dtype, device="cuda")
    tree.adjust_logits(wide[:, :1100], out=left[:, 3:1103])
    assert (left[:, :3] == 9).all() and (left[:, 1103:] == 9).all()


def test_adjust_in_a_graph_and_refusals(tree):
    z = torch.randn((4, 300), device="cuda")
    hist, n = dev(np.arange(20).reshape(2, 10)), dev([10, 4])
    f = torch.full((2,), 0.5, device="cuda")
    want = tree.adjust_logits(z, hist, n, frequency=f)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = tree.adjust_logits(z, hist, n, frequency=f)
    got.zero_()
    graph.replay()
    assert torch.equal(got, want)
    assert tree.adjust_logits(z[:0]).shape == (0, 300)
    i = dev([[1, 2]] * 2)
    for kw in (dict(history=hist), dict(hist_len=n), dict(history=hist, hist_len=n.long()), dict(bias_ids=i), dict(bias=f), dict(tokens=i),
               dict(repetition=f.double()), dict(frequency=torch.ones(3, device="cuda")), dict(allowed=dev(np.zeros((4, 9)))),
               dict(allowed=dev(np.zeros((2, 10)))), dict(out=torch.empty(4, 301, device="cuda")), dict(out=torch.empty(4, 300)),
               dict(tokens=i, mask=torch.zeros((2, 2, 2), dtype=torch.int64, device="cuda"))):
        with pytest.raises(ValueError):
            tree.adjust_logits(z, **kw)
    from paper_2504_18583_gb300.pard import PardError
    many = torch.zeros((1, 2048), device="cuda")
    with pytest.raises(PardError):
        tree.adjust_logits(z, bias_ids=many.int(), bias=many)
    with pytest.raises(ValueError):
        tree.adjust_logits(z.double())


# ---- as they are used together ---------------------------------------------------------
@pytest.mark.parametrize("eight", [False, True])
def test_a_prompt_in_pieces_then_tokens(tree, eight):
    """A prompt read in uneven pieces and token by token gives each position what reading it whole does: the cache's
    entries are the same bits, and outputs agree to their roundings (u |o| + 2 u sum w |v| each)."""
    Hq, Hkv, hd, T = 8, 2, 64, 333
    g = torch.Generator(device="cuda").manual_seed(1)
    qkv = torch.randn((2 * T, (Hq + 2 * Hkv) * hd), generator=g, device="cuda").to(BF)
    table = np.random.RandomState(0).permutation(50)[:44].reshape(2, 22)
    gains = [(1 + 0.2 * torch.randn(hd, generator=g, device="cuda")).to(BF) for _ in range(2)]
    freq, amp = tree.rope_frequencies(hd, 1e4)

    def read(pieces):
        """[2 T, Hq, hd] outputs of both sequences read in the pieces, and the cache."""
        if eight:
            k, v, ks, vs = tree.quantized_cache(50, Hkv, hd)
        else:
            k, v = (torch.zeros((50, Hkv, PAGE, hd), dtype=BF, device="cuda") for _ in range(2))
            ks = vs = None
        out, done = torch.empty((2, T, Hq, hd), dtype=BF, device="cuda"), np.zeros(2, int)
        for new in pieces:
            rows = np.concatenate([b * T + done[b] + np.arange(new[b]) for b in range(2)])
            pos = np.concatenate([done[b] + np.arange(new[b]) for b in range(2)])
            slots = np.concatenate([table[b, (done[b] + np.arange(new[b])) // PAGE] * PAGE + (done[b] + np.arange(new[b])) % PAGE for b in range(2)])
            q = tree.qk_norm_rope(qkv[dev(rows, torch.int64)], Hq, Hkv, dev(pos), dev(slots, torch.int64), k, v, freq, *gains, amplitude=amp,
                                  k_scale=ks, v_scale=vs)
            o = tree.chunk_attention(q, k, v, dev(table), dev(np.cumsum([0] + list(new))), dev(done), window=150, sinks=4, k_scale=ks, v_scale=vs)
            at = 0
            for b in range(2):
                out[b, done[b]:done[b] + new[b]] = o[at:at + new[b]]
                at += new[b]
                done[b] += new[b]
        assert (done == T).all()
        return out, (k.view(torch.uint8), v.view(torch.uint8))

    whole, cache = read([(T, T)])
    pieces, cache2 = read([(100, 1), (1, 231), (200, 1), (31, 1), (1, T - 234)])
    assert all(torch.equal(a, b) for a, b in zip(cache, cache2))
    u = ROUND[BF]
    # |v| is below 6, so sum w |v| is; typical outputs are far smaller
    assert ((whole.double() - pieces.double()).abs() <= 2 * u * whole.double().abs() + 4 * u * 6).all()
    assert float((whole.double() - pieces.double()).abs().mean()) < u


def test_adjust_then_sample_over_a_tree(tree):
    """The nodes of two trees: rows adjusted with their branches, then drawn; a forbidden token is never drawn, and the
    token of a greedy draw is the adjusted row's largest."""
    rs = np.random.RandomState(3)
    B, N, V = 2, 9, 700
    parents = np.array([[-1] + [int(rs.randint(0, i)) for i in range(1, N)] for _ in range(B)])
    mask, _, _ = tree.tree_plan(dev(parents), dev([N, N]), dev([20, 3]), dev(np.arange(8).reshape(2, 4)), 8)
    tokens = rs.randint(0, V, (B, N))
    z = torch.randn((B * N, V), device="cuda") * 3
    allowed = words_of(rs.rand(B * N, V) < 0.1)
    kw = dict(hist=rs.randint(0, V, (B, 30)), hist_len=np.array([30, 12]), rep=[1.2, 1.1], freq=[0.3, 0.2], pres=[0.1, 0.4], allowed=allowed,
              tokens=tokens, mask=mask.cpu().numpy().view(np.uint64))
    got = check_adjust(tree, z, N, **kw)
    token, _ = tree.sample(got, torch.rand(B * N, device="cuda"), temperature=torch.full((B * N,), 0.9, device="cuda"))
    bits = np.unpackbits(allowed.view(np.uint8), axis=1, bitorder="little")
    assert all(bits[r, t] for r, t in enumerate(token.tolist()))
    token, _ = tree.sample(got, torch.zeros(B * N, device="cuda"), temperature=torch.zeros(B * N, device="cuda"))
    assert token.tolist() == got.argmax(1).tolist()
