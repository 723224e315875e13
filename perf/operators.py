"""The operators of the decode step for a tree of drafted tokens, as measured cases.

``tree_plan`` turns parent links into masks, positions and cache slots;
``qk_norm_rope`` norms and rotates queries and keys and writes the paged
cache; ``tree_attention`` attends over the cache and a node's ancestors;
``sample`` draws one token a row; ``tree_commit`` walks the sampled tokens
down the tree and compacts the accepted path's rows in the cache.

``run`` computes a case in elementary torch operations in 32 bits, or, where
``own`` is set, by the library's calls.  Model shapes are the repository's:
8B (32 query and 8 key/value heads of 128), 1B (32 / 8 of 64), 70B (64 / 8 of
128), vocabularies of 128256 and 2048; pages hold 16 tokens.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

PAGE = 16
HEADS = {"8b": (32, 8, 128), "1b": (32, 8, 64), "70b": (64, 8, 128)}
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
THETA = 500000.0
VOCAB = 128256
# the batch-16 configuration's prompt lengths, uniform in [128, 2048]
LENS16 = "1922,1532,161,1596,1020,1843,1698,1705,940,247,232,657,267,785,660,691"
BITS = 40  # fractional bits of the sampler's integer weights


def listed():
    def plan(name, **kw):
        return dict(name=name, op="plan", **kw)

    def rope(name, **kw):
        return dict(name=name, op="rope", **kw)

    def attn(name, **kw):
        return dict(name=name, op="attn", **kw)

    def sample(name, **kw):
        return dict(name=name, op="sample", **kw)

    def commit(name, **kw):
        return dict(name=name, op="commit", **kw)

    return [
        # the plan of one sequence's small tree (pure latency), and of a full batch of the widest trees
        plan("plan_b1_n29", lens="512", nodes="29", width=29),
        plan("plan_b64_n256", lens=_spread(64, 37, 4000), nodes=_spread(64, 100, 256), width=256),
        # a verify pass of 9 rows of the 8B shape (latency), and a long prompt of odd length at scaled positions
        rope("rope_8b_9rows", model="8b", dtype="bf16", tokens=9, start=512, rot=128, interleaved=False, norm=True,
             scaling="none"),
        rope("rope_8b_prompt_8191", model="8b", dtype="bf16", tokens=8191, start=100000, rot=128, interleaved=False,
             norm=True, scaling="yarn"),
        # one token of one sequence: the autoregressive step's attention at the headline context
        attn("attn_8b_b1_n1_ctx512", model="8b", dtype="bf16", lens="512", nodes="1", width=1),
        # the batch-16 configuration's ragged contexts with trees of 17 to 29 nodes
        attn("attn_8b_b16_n29_ragged", model="8b", dtype="bf16", lens=LENS16, nodes=_spread(16, 17, 29), width=29),
        # 70B heads, wide trees at the 4096-token context: the most arithmetic for a byte of cache
        attn("attn_70b_b8_n64_ctx4096", model="70b", dtype="fp16", lens=",".join(["4096"] * 8),
             nodes=",".join(["64"] * 8), width=64),
        # long contexts: two sequences, small heads, a tree that is no round number
        attn("attn_1b_b2_n13_ctx65k", model="1b", dtype="bf16", lens="65521,50001", nodes="13,11", width=13),
        # the draw of one sequence's next token, and of every node of a batch of trees
        sample("sample_1x128256", rows=1, vocab=VOCAB, dtype="fp32", mode="mix"),
        sample("sample_464x128256", rows=464, vocab=VOCAB, dtype="fp32", mode="mix"),
        # one sequence's accepted path, and a batch of wide trees, over 32 layers
        commit("commit_8b_b1_n29", model="8b", dtype="bf16", layers=32, lens="512", nodes="29", width=29),
        commit("commit_8b_b16_n64", model="8b", dtype="bf16", layers=32, lens=_spread(16, 37, 700),
               nodes=_spread(16, 40, 64), width=64),
    ]


def _spread(count, lo, hi):
    """`count` whole numbers over [lo, hi], out of order, as text."""
    step = 0.6180339887498949
    return ",".join(str(lo + int((hi - lo + 1) * ((0.37 + i * step) % 1.0))) for i in range(count))


def _ints(text):
    return [int(x) for x in text.split(",")]


def draw(rng):
    def log_int(lo, hi):
        return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    op = rng.choice(["plan", "rope", "attn", "attn", "attn", "sample", "sample", "commit"])
    if op == "plan":
        batch, width = log_int(1, 64), log_int(1, 256)
        return dict(op="plan", lens=",".join(str(log_int(1, 4000)) for _ in range(batch)),
                    nodes=",".join(str(rng.randint(max(1, width // 2), width)) for _ in range(batch)), width=width)
    if op == "rope":
        model = rng.choice(["8b", "1b", "70b"])
        hd = HEADS[model][2]
        return dict(op="rope", model=model, dtype=rng.choice(["bf16", "fp16"]),
                    tokens=log_int(1, 8191 if model != "70b" else 4500), start=log_int(1, 120000),
                    rot=rng.choice([hd, hd, hd // 2, hd // 4]), interleaved=rng.random() < 0.5,
                    norm=rng.random() < 0.7, scaling=rng.choice(["none", "linear", "ntk", "parts", "yarn"]))
    if op == "attn":
        model = rng.choice(["8b", "1b", "70b"])
        batch, width = log_int(1, 16), log_int(1, 64)
        Hq, _, hd = HEADS[model]
        # no more keys than the long-context case, no more products than the widest trees
        top = max(64, min(65000, 110000 // batch, int(6.5e10 / (4 * hd * Hq * batch * width))))
        return dict(op="attn", model=model, dtype=rng.choice(["bf16", "fp16"]),
                    lens=",".join(str(log_int(max(1, top // 30), top)) for _ in range(batch)),
                    nodes=",".join(str(rng.randint(max(1, width // 2), width)) for _ in range(batch)), width=width)
    if op == "sample":
        vocab = log_int(2048, VOCAB)
        return dict(op="sample", rows=log_int(1, 464), vocab=vocab, dtype=rng.choice(["fp32", "bf16", "fp16"]),
                    mode=rng.choice(["mix", "topp", "topk", "plain"]))
    batch, width = log_int(1, 16), log_int(2, 64)
    return dict(op="commit", model=rng.choice(["8b", "1b"]), dtype=rng.choice(["bf16", "fp16"]),
                layers=rng.choice([4, 16, 32]), lens=",".join(str(log_int(1, 700)) for _ in range(batch)),
                nodes=",".join(str(rng.randint(max(1, width // 2), width)) for _ in range(batch)), width=width)


# ---- inputs -----------------------------------------------------------------
def _dev(a, dtype):
    return torch.tensor(np.asarray(a), dtype=dtype, device="cuda")


def _tree(rs, n):
    """Parent links of a tree of n nodes whose first is the root: most candidates hang on a recent node."""
    parents = np.full(n, -1, np.int64)
    for i in range(1, n):
        parents[i] = rs.randint(max(0, i - 12), i)
    return parents


def _sequences(case, rs, extra_pages=3):
    """Trees, lengths and a page table over a pool of shuffled pages."""
    lens, nodes, width = _ints(case["lens"]), _ints(case["nodes"]), case["width"]
    parents = np.full((len(lens), width), -1, np.int64)
    for b, n in enumerate(nodes):
        parents[b, :n] = _tree(rs, n)
    need = [-(-(l + n) // PAGE) for l, n in zip(lens, nodes)]
    order = rs.permutation(sum(need) + extra_pages)
    table, at = np.zeros((len(lens), max(need)), np.int64), 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return dict(parents=_dev(parents, torch.int32), nodes=_dev(nodes, torch.int32), lens=_dev(lens, torch.int32),
                table=_dev(table, torch.int32), n_pages=int(order.size), host=(parents, lens, nodes))


def _ancestors(parents, nodes):
    """[B, N, N] truth: column j is row i or one of its ancestors; rows past a sequence's nodes are empty."""
    B, N = parents.shape
    at = torch.arange(N, device=parents.device)
    live = at[None] < nodes[:, None]
    reach = ((parents[:, :, None] == at) | (at[:, None] == at)).float()
    for _ in range(max(1, (N - 1).bit_length())):  # each product doubles the links that are followed
        reach = (reach @ reach > 0).float()
    return (reach > 0) & live[:, :, None] & live[:, None, :]


def _pack(rows):
    """[B, N, N] truth -> [B, N, ceil(N / 64)] words of 64 columns, the lowest column in the lowest bit."""
    B, N, _ = rows.shape
    W = -(-N // 64)
    bits = torch.nn.functional.pad(rows, (0, 64 * W - N)).view(B, N, W, 64).to(torch.int64)
    return (bits << torch.arange(64, device=rows.device)).sum(-1)


def _rope_plan(case):
    """Frequencies (radians a position) of the rotated pairs and the amplitude, for the case's scaling."""
    R, i = case["rot"], np.arange(case["rot"] // 2, dtype=np.float64)
    freq = THETA ** (-2.0 * i / R)
    kind, factor, first = case["scaling"], 8.0, 8192.0  # scaled to 8 times the 8192 positions of the base
    amp = 1.0
    if kind == "linear":
        freq = freq / factor
    elif kind == "ntk":
        freq = (THETA * factor ** (R / (R - 2.0))) ** (-2.0 * i / R)
    elif kind == "parts":
        turns = first * freq / (2 * math.pi)
        keep = np.clip((turns - 1.0) / (4.0 - 1.0), 0.0, 1.0)
        freq = freq * keep + freq / factor * (1 - keep)
    elif kind == "yarn":
        dim = lambda turns: R * math.log(first / (turns * 2 * math.pi)) / (2 * math.log(THETA))  # noqa: E731
        lo, hi = max(math.floor(dim(32.0)), 0), min(math.ceil(dim(1.0)), R - 1)
        keep = 1.0 - np.clip((i - lo) / max(hi - lo, 0.001), 0.0, 1.0)
        freq = freq * keep + freq / factor * (1 - keep)
        amp = 0.1 * math.log(factor) + 1.0
    return torch.tensor(freq.astype(np.float32), device="cuda"), float(np.float32(amp))


def prepare(case, seed):
    rs = np.random.RandomState(seed % (1 << 31))
    g = torch.Generator(device="cuda").manual_seed(seed)
    op = case["op"]
    s = dict(op=op)
    if op == "sample":
        R, V = case["rows"], case["vocab"]
        # a broad bell with a few dozen tokens that stand out, as next-token logits have
        z = 2.0 * torch.randn((R, V), generator=g, device="cuda")
        hot = torch.randint(0, V, (R, 64), generator=g, device="cuda")
        lift = 14.0 * torch.rand((R, 64), generator=g, device="cuda")
        s["logits"] = z.scatter_add(1, hot, lift).to(DTYPES[case["dtype"]])
        s["u"] = torch.rand(R, generator=g, device="cuda")
        mode = case["mode"]
        T = rs.uniform(0.6, 1.3, R)
        k, p, m = np.zeros(R, np.int64), np.ones(R), np.zeros(R)
        if mode in ("mix", "topk"):
            k = np.where(rs.rand(R) < (0.5 if mode == "mix" else 2), rs.randint(1, 200, R), 0)
        if mode in ("mix", "topp"):
            p = np.where(rs.rand(R) < (0.7 if mode == "mix" else 2), rs.uniform(0.5, 0.99, R), 1.0)
        if mode == "mix":
            m = np.where(rs.rand(R) < 0.3, rs.uniform(0.005, 0.2, R), 0.0)
            T = np.where(rs.rand(R) < 0.1, 0.0, T)
        if R == 1:  # the one row takes every cut
            T, k, p, m = T * 0 + 0.8, k * 0 + 50, p * 0 + 0.95, m * 0 + 0.01
            if mode in ("topp", "plain"):
                k, m = k * 0, m * 0
            if mode in ("topk", "plain"):
                p, m = p * 0 + 1.0, m * 0
        s.update(temperature=_dev(T, torch.float32), top_k=_dev(k, torch.int32), top_p=_dev(p, torch.float32),
                 min_p=_dev(m, torch.float32))
        return s
    if op == "rope":
        Hq, Hkv, hd = HEADS[case["model"]]
        T, dt = case["tokens"], DTYPES[case["dtype"]]
        n_pages = -(-T // PAGE) + 2
        order = torch.randperm(n_pages, generator=g, device="cuda")
        at = torch.arange(T, device="cuda")
        s.update(Hq=Hq, Hkv=Hkv, hd=hd, interleaved=case["interleaved"], rot=case["rot"], eps=1e-5,
                 qkv=(1.5 * torch.randn((T, (Hq + 2 * Hkv) * hd), generator=g, device="cuda")).to(dt),
                 pos=(at + case["start"]).to(torch.int32), slots=order[at // PAGE] * PAGE + at % PAGE)
        s["freq"], s["amp"] = _rope_plan(case)
        for name in ("q_gain", "k_gain"):
            s[name] = (1 + 0.2 * torch.randn(hd, generator=g, device="cuda")).to(dt) if case["norm"] else None
        for name in ("k_cache", "v_cache"):
            s[name] = torch.zeros((n_pages, Hkv, PAGE, hd), dtype=dt, device="cuda")
        return s
    s.update(_sequences(case, rs))
    parents, lens, nodes = s.pop("host")
    if op == "attn":
        Hq, Hkv, hd = HEADS[case["model"]]
        dt = DTYPES[case["dtype"]]
        B, N = parents.shape
        s["mask"] = _pack(_ancestors(s["parents"].long(), s["nodes"].long()))
        # scores with a spread of about 1.5, so that some keys stand out of a long context
        s["q"] = (1.5 * torch.randn((B, N, Hq, hd), generator=g, device="cuda")).to(dt)
        for name in ("k_cache", "v_cache"):
            s[name] = torch.randn((s["n_pages"], Hkv, PAGE, hd), generator=g, device="cuda").to(dt)
    if op == "commit":
        Hq, Hkv, hd = HEADS[case["model"]]
        B, N = parents.shape
        tokens, sampled = rs.randint(0, VOCAB, (B, N)), rs.randint(0, VOCAB, (B, N))
        for b, n in enumerate(nodes):  # the target agrees with one of a node's children four times in five
            for i in range(n):
                kids = np.flatnonzero(parents[b, :n] == i)
                if len(kids) and rs.rand() < 0.8:
                    sampled[b, i] = tokens[b, kids[rs.randint(len(kids))]]
        s.update(tokens=_dev(tokens, torch.int32), sampled=_dev(sampled, torch.int32))
        s["pool"] = torch.randn((case["layers"], 2, s["n_pages"], Hkv, PAGE, hd), generator=g, device="cuda",
                                dtype=DTYPES[case["dtype"]])
    return s


# ---- one pass ---------------------------------------------------------------
def run(s):
    if own:
        from paper_2504_18583_gb300 import tree
        return _own(s, tree)
    return _PLAIN[s["op"]](s)


def _own(s, tree):
    op = s["op"]
    if op == "plan":
        return tree.tree_plan(s["parents"], s["nodes"], s["lens"], s["table"], s["n_pages"])
    if op == "rope":
        q = tree.qk_norm_rope(s["qkv"], s["Hq"], s["Hkv"], s["pos"], s["slots"], s["k_cache"], s["v_cache"],
                              s["freq"], q_gain=s["q_gain"], k_gain=s["k_gain"], eps=s["eps"],
                              interleaved=s["interleaved"], amplitude=s["amp"])
        return q, s["k_cache"], s["v_cache"]
    if op == "attn":
        return tree.tree_attention(s["q"], s["k_cache"], s["v_cache"], s["table"], s["lens"], s["nodes"], s["mask"])
    if op == "sample":
        return tree.sample(s["logits"], s["u"], s["temperature"], s["top_k"], s["top_p"], s["min_p"])
    accept, emitted, length = tree.tree_commit(s["sampled"], s["tokens"], s["parents"], s["nodes"], s["lens"],
                                               s["table"], s["pool"])
    return accept, emitted, length, s["pool"]


def _plain_plan(s):
    lens, nodes, table = s["lens"].long(), s["nodes"].long(), s["table"].long()
    reach = _ancestors(s["parents"].long(), nodes)
    B, N = s["parents"].shape
    at = torch.arange(N, device="cuda")
    live = at[None] < nodes[:, None]
    pos = torch.where(live, lens[:, None] + reach.sum(-1) - 1, 0)
    where = lens[:, None] + at[None]
    page = torch.gather(table, 1, (where // PAGE).clamp(max=table.shape[1] - 1))
    slots = torch.where(live & (where // PAGE < table.shape[1]), page * PAGE + where % PAGE, -1)
    return _pack(reach), pos.to(torch.int32), slots


def _rotate(x, cos, sin, rot, interleaved):
    """Rotates the first `rot` entries of the last dimension; cos and sin: [T, 1, rot / 2]."""
    head, rest = x[..., :rot], x[..., rot:]
    if interleaved:
        a, b = head[..., 0::2], head[..., 1::2]
        head = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    else:
        a, b = head[..., :rot // 2], head[..., rot // 2:]
        head = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    return torch.cat([head, rest], -1)


def _plain_rope(s):
    Hq, Hkv, hd, dt = s["Hq"], s["Hkv"], s["hd"], s["qkv"].dtype
    x = s["qkv"].float().view(-1, Hq + 2 * Hkv, hd)
    q, k, v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    # angles in turns of 2^-40, so that a far position does not wear the frequency's bits away
    turn = (s["freq"].double() / (2 * math.pi) * 2.0 ** 40).round().long()
    phase = (s["pos"].long()[:, None] * turn[None]) & (2 ** 40 - 1)
    angle = (phase.float() * (2 * math.pi / 2.0 ** 40))[:, None]
    cos, sin = s["amp"] * torch.cos(angle), s["amp"] * torch.sin(angle)
    if s["q_gain"] is not None:
        q = q * torch.rsqrt(q.square().mean(-1, keepdim=True) + s["eps"]) * s["q_gain"].float()
        k = k * torch.rsqrt(k.square().mean(-1, keepdim=True) + s["eps"]) * s["k_gain"].float()
    q = _rotate(q, cos, sin, s["rot"], s["interleaved"]).to(dt)
    k = _rotate(k, cos, sin, s["rot"], s["interleaved"]).to(dt)
    page, at = s["slots"] // PAGE, s["slots"] % PAGE
    s["k_cache"][page, :, at] = k
    s["v_cache"][page, :, at] = v.to(dt)
    return q, s["k_cache"], s["v_cache"]


def _keys(cache, table):
    """[B, Hkv, P * 16, hd] of a paged cache."""
    B, P = table.shape
    x = cache[table.long()]
    return x.permute(0, 2, 1, 3, 4).reshape(B, x.shape[2], P * PAGE, x.shape[4])


def _allowed(mask, lens, nodes, n_keys):
    """[B, N, n_keys] truth: the context, and the tree's keys whose bit is set."""
    B, N, W = mask.shape
    bits = (mask[..., None] >> torch.arange(64, device=mask.device)) & 1
    bits = bits.view(B, N, W * 64) == 1
    j = torch.arange(n_keys, device=mask.device)[None] - lens[:, None]
    tree = torch.gather(bits, 2, j.clamp(0, W * 64 - 1)[:, None].expand(B, N, n_keys))
    live = torch.arange(N, device=mask.device)[None] < nodes[:, None]
    return ((j < 0)[:, None] | (tree & ((j >= 0) & (j < nodes[:, None]))[:, None])) & live[:, :, None]


def _plain_attn(s):
    B, N, Hq, hd = s["q"].shape
    lens, nodes = s["lens"].long(), s["nodes"].long()
    k, v = _keys(s["k_cache"], s["table"]).float(), _keys(s["v_cache"], s["table"]).float()
    Hkv, n_keys = k.shape[1], k.shape[2]
    v = torch.where((torch.arange(n_keys, device="cuda")[None] < (lens + nodes)[:, None])[:, None, :, None], v, 0.0)
    q = s["q"].float().view(B, N, Hkv, Hq // Hkv, hd).permute(0, 2, 1, 3, 4).reshape(B, Hkv, -1, hd)
    score = (q @ k.transpose(2, 3)).mul_(hd ** -0.5).view(B, Hkv, N, -1, n_keys)
    score = score.masked_fill_(~_allowed(s["mask"], lens, nodes, n_keys)[:, None, :, None], float("-inf"))
    top = score.amax(-1, keepdim=True)
    w = score.sub_(torch.where(top > float("-inf"), top, 0.0)).exp_()
    total = w.sum(-1, keepdim=True)
    o = (w.view(B, Hkv, -1, n_keys) @ v).view(B, Hkv, N, -1, hd) / torch.where(total > 0, total, 1.0)
    return o.permute(0, 2, 1, 3, 4).reshape(B, N, Hq, hd).to(s["q"].dtype)


def _plain_sample(s):
    z = s["logits"].float()
    z = torch.where(torch.isnan(z), float("-inf"), z)
    R, V = z.shape
    top = z.amax(1, keepdim=True)
    T = s["temperature"][:, None]
    x = torch.where(z == top, 0.0, (z - top) / torch.where(T > 0, T, 1.0))
    w = torch.where(z == float("-inf"), 0.0, torch.exp(x))
    whole = (w * 2.0 ** BITS).round().long()  # sums of whole numbers have no order
    zs, order = torch.sort(z, dim=1, descending=True, stable=True)
    ws = torch.gather(whole, 1, order)
    rank = torch.arange(V, device="cuda")[None]
    k = s["top_k"].long()[:, None]
    keep = rank < torch.where(k > 0, k, V)
    cut = torch.where(keep, ws, 0)
    upto = cut.cumsum(1)
    bar = s["top_p"].double()[:, None] * upto[:, -1:].double()
    keep &= ((upto - cut).double() < bar) | (rank == 0)
    keep &= (torch.gather(w, 1, order) >= s["min_p"][:, None]) | (rank == 0)
    keep = torch.zeros_like(keep).scatter_(1, order, keep)
    kept = torch.where(keep, whole, 0)
    upto = kept.cumsum(1)
    total = upto[:, -1:]
    token = (upto.double() <= s["u"].double()[:, None] * total.double()).sum(1).clamp(max=V - 1)
    won = torch.gather(whole, 1, token[:, None])
    logp = -torch.log1p((total - won).float() / won.float())[:, 0]
    first = (z == top).to(torch.int8).argmax(1)
    greedy, empty = s["temperature"] <= 0, top[:, 0] == float("-inf")
    token = torch.where(empty, -1, torch.where(greedy, first, token))
    logp = torch.where(empty, float("-inf"), torch.where(greedy, 0.0, logp))
    return token.to(torch.int32), logp


def _walk(sampled, tokens, parents, nodes):
    """Which nodes the sampled tokens lead through: [B, N] truth."""
    B, N = parents.shape
    at = torch.arange(N, device=parents.device)
    live = at[None] < nodes[:, None]
    said = torch.gather(sampled, 1, parents.clamp(min=0))  # what the parent's row drew
    hit = (parents >= 0) & (said == tokens) & live
    twin = (parents[:, :, None] == parents[:, None, :]) & hit[:, None, :] & (at[None, :] < at[:, None])
    hit &= ~twin.any(-1)  # the lowest of the children that match
    reach = _ancestors(parents, nodes)
    return (~reach | hit[:, None, :] | (at == 0)).all(-1) & live & (reach[:, :, 0])


def _plain_commit(s):
    parents, nodes, lens, table = s["parents"].long(), s["nodes"].long(), s["lens"].long(), s["table"].long()
    B, N = parents.shape
    on = _walk(s["sampled"], s["tokens"], parents, nodes)
    count = on.sum(1)
    j = torch.arange(N, device="cuda")
    path = torch.sort(torch.where(on, j, N), 1).values
    valid = path < N
    path = path.clamp(max=N - 1)
    emitted = torch.where(valid, torch.gather(s["sampled"].long(), 1, path), -1)

    def slot(where):
        return torch.gather(table, 1, (where // PAGE).clamp(max=table.shape[1] - 1)), where % PAGE

    sp, so = slot(lens[:, None] + path)
    dp, do = slot(lens[:, None] + j[None])
    moves = valid & (path != j)
    rows = s["pool"][:, :, sp[moves], :, so[moves]]
    s["pool"][:, :, dp[moves], :, do[moves]] = rows
    return ((count - 1).clamp(min=0).to(torch.int32), emitted.to(torch.int32), (lens + count).to(torch.int32), s["pool"])


_PLAIN = {"plan": _plain_plan, "rope": _plain_rope, "attn": _plain_attn, "sample": _plain_sample,
          "commit": _plain_commit}


# ---- what a pass cannot do without -------------------------------------------
def work(case):
    op = case["op"]
    if op == "sample":
        size = 4 if case["dtype"] == "fp32" else 2
        n = case["rows"] * case["vocab"]
        return dict(bytes=n * size + case["rows"] * 28, flops=4 * n)
    if op == "rope":
        Hq, Hkv, hd = HEADS[case["model"]]
        n = case["tokens"] * (Hq + 2 * Hkv) * hd
        return dict(bytes=4 * n + 12 * case["tokens"], flops=8 * n)
    lens, nodes, N = _ints(case["lens"]), _ints(case["nodes"]), case["width"]
    B, W = len(lens), -(-N // 64)
    if op == "plan":
        return dict(bytes=B * N * (4 + 8 * W + 4 + 8) + 8 * B, flops=sum(nodes))
    Hq, Hkv, hd = HEADS[case["model"]]
    if op == "attn":
        keys = sum(l + n for l, n in zip(lens, nodes))
        return dict(bytes=4 * keys * Hkv * hd + 2 * Hq * hd * (sum(nodes) + B * N) + 8 * W * sum(nodes),
                    flops=4 * hd * Hq * sum(n * (l + 1) for l, n in zip(lens, nodes)))
    # the accepted rows depend on the draws: about three a sequence of this many nodes
    moved = sum(min(3, max(0, n - 1)) for n in nodes)
    return dict(bytes=4 * 2 * case["layers"] * Hkv * hd * moved + 12 * sum(nodes), flops=sum(nodes))


# ---- the operators' definitions in 64 bits -----------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "rope":
        return _exact_rope(s)
    if case["op"] == "attn":
        return _exact_attn(s)
    if case["op"] == "sample":
        return _exact_sample(s)
    return None  # whole numbers, and rows that are moved as they are


def _exact_rope(s):
    Hq, Hkv, hd, half = s["Hq"], s["Hkv"], s["hd"], s["rot"] // 2
    x = s["qkv"].cpu().double().numpy().reshape(-1, Hq + 2 * Hkv, hd)
    angle = s["pos"].cpu().double().numpy()[:, None] * s["freq"].cpu().double().numpy()[None]
    turn = (s["amp"] * np.exp(1j * angle))[:, None]
    heads = []
    for lo, hi, gain in ((0, Hq, s["q_gain"]), (Hq, Hq + Hkv, s["k_gain"])):
        y = x[:, lo:hi].copy()
        if gain is not None:
            y = y / np.sqrt(np.mean(y * y, -1, keepdims=True) + s["eps"]) * gain.cpu().double().numpy()
        a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if s["interleaved"] else (slice(0, half), slice(half, 2 * half))
        c = (y[..., a] + 1j * y[..., b]) * turn
        y[..., a], y[..., b] = c.real, c.imag
        heads.append(y)
    out = [torch.from_numpy(heads[0])]
    slots = s["slots"].cpu().numpy()
    for rows in (heads[1], x[:, Hq + Hkv:]):
        cache = np.zeros(tuple(s["k_cache"].shape))
        cache[slots // PAGE, :, slots % PAGE] = rows
        out.append(torch.from_numpy(cache))
    return tuple(out)


def _exact_attn(s):
    """Sequence by sequence over the keys that each has, with the largest score taken out of the exponentials."""
    B, N, Hq, hd = s["q"].shape
    if B * N * Hq * s["table"].shape[1] * PAGE > 3e9:
        return None
    Hkv = s["k_cache"].shape[1]
    out = torch.zeros((B, N, Hq, hd), dtype=torch.float64, device="cuda")
    words = s["mask"].cpu().numpy().view(np.uint64)
    for b in range(B):
        L, n = int(s["lens"][b]), int(s["nodes"][b])
        flat = s["table"][b, :-(-(L + n) // PAGE)].long()
        K = s["k_cache"][flat].transpose(0, 1).reshape(Hkv, -1, hd)[:, :L + n].double()
        V = s["v_cache"][flat].transpose(0, 1).reshape(Hkv, -1, hd)[:, :L + n].double()
        sees = np.unpackbits(words[b, :n].view(np.uint8), axis=-1, bitorder="little")[:, :n].astype(bool)
        bias = torch.zeros((n, L + n), dtype=torch.float64, device="cuda")
        bias[:, L:] = torch.from_numpy(np.where(sees, 0.0, -np.inf)).to("cuda")
        for h in range(Hq):
            a = s["q"][b, :n, h].double() @ K[h // (Hq // Hkv)].T / math.sqrt(hd) + bias
            out[b, :n, h] = torch.softmax(a, -1) @ V[h // (Hq // Hkv)]
    return out


def _exact_sample(s):
    R = s["logits"].shape[0]
    token, logp = torch.full((R,), -1, dtype=torch.int32), torch.full((R,), float("-inf"), dtype=torch.float64)
    at = {n: s[n].cpu().double().numpy() for n in ("u", "temperature", "top_k", "top_p", "min_p")}
    for r in range(R):
        z = s["logits"][r].double().cpu().numpy()
        if at["temperature"][r] <= 0:
            token[r], logp[r] = int(np.argmax(z)), 0.0
            continue
        w = np.exp((z - z.max()) / at["temperature"][r])
        order = np.argsort(-z, kind="stable")
        k = int(at["top_k"][r])
        order = order[:k] if k > 0 else order
        before = np.cumsum(w[order]) - w[order]
        fits = (before < at["top_p"][r] * w[order].sum()) & (w[order] >= at["min_p"][r])
        fits[0] = True
        kept = np.sort(order[fits])
        upto = np.cumsum(w[kept])
        i = min(int(np.searchsorted(upto, at["u"][r] * upto[-1], side="right")), len(kept) - 1)
        token[r], logp[r] = int(kept[i]), -math.log1p((upto[-1] - w[kept[i]]) / w[kept[i]])
    return token, logp
