"""Operators of a serving loop around the decode step, as measured cases.

``chunk_attention`` attends for a chunk of new tokens a sequence (a piece of a
prompt, or the next token) over the paged cache, with a sliding window and a
few first tokens that stay visible; the cache holds 16-bit entries, or 8-bit
ones with a power of two for each token and head.  ``qk_norm_rope`` with an
8-bit cache norms and rotates queries and keys and quantises keys and values as
it writes them.  ``adjust_logits`` applies what a request asks of its logits:
penalties for tokens that were there, biases, and a grammar's mask.

``run`` computes a case in elementary torch operations in 32 bits, or, where
``own`` is set, by the library's calls.  Model shapes are the repository's:
8B (32 query and 8 key/value heads of 128), 1B (32 / 8 of 64), 70B (64 / 8 of
128), a vocabulary of 128256; pages hold 16 tokens.
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
TOP8 = 448.0  # largest finite value of e4m3
# new tokens of a batch in which prompts are read in pieces while others decode
MIXED = "700,1,1,513,1,1,129,1,1,1,1,64,1,1,17,1"


def listed():
    def chunk(name, **kw):
        return dict(name=name, op="chunk", **kw)

    def write(name, **kw):
        return dict(name=name, op="write", **kw)

    def adjust(name, **kw):
        return dict(name=name, op="adjust", **kw)

    return [
        # the next token of one sequence that keeps a window of 2048 and its first four tokens (latency)
        chunk("chunk_8b_1token_window2048", model="8b", dtype="bf16", cache="16", new="1", ctx="20011", window=2048, sinks=4),
        # four sequences, a piece of their prompts each behind what was read before
        chunk("chunk_8b_b4_512_ragged", model="8b", dtype="bf16", cache="16", new="512,512,512,400", ctx="1024,0,3600,2111",
              window=0, sinks=0),
        # a whole prompt of odd length at once
        chunk("chunk_8b_prompt_8191", model="8b", dtype="bf16", cache="16", new="8191", ctx="0", window=0, sinks=0),
        # a large piece of a long document, 70B heads: the most products
        chunk("chunk_70b_2048_ctx30k", model="70b", dtype="fp16", cache="16", new="2048", ctx="30000", window=0, sinks=0),
        # pieces of prompts and single tokens in one batch, small heads, window and first tokens
        chunk("chunk_1b_b16_mixed_window", model="1b", dtype="bf16", cache="16", new=MIXED, ctx=_spread(16, 300, 9000),
              window=1024, sinks=4),
        # the next token of 32 sequences over an 8-bit cache: nothing but reading it
        chunk("chunk_8b_b32_1token_8bit", model="8b", dtype="bf16", cache="8", new=",".join(["1"] * 32),
              ctx=_spread(32, 500, 16000), window=0, sinks=0),
        # a piece of a prompt over an 8-bit cache
        chunk("chunk_8b_1000_ctx16k_8bit", model="8b", dtype="bf16", cache="8", new="1000", ctx="16001", window=0, sinks=0),
        # the rows of one batch's next tokens into the 8-bit cache (latency), and a whole prompt's
        write("write_8b_16rows", model="8b", dtype="bf16", tokens=16, start=512, rot=128, interleaved=False, norm=True),
        write("write_8b_prompt_8191", model="8b", dtype="bf16", tokens=8191, start=0, rot=128, interleaved=False, norm=True),
        # one request's next token with everything asked for at once
        adjust("adjust_1x128256", batch=1, width=1, vocab=VOCAB, dtype="fp32", history=2000, biases=20, grammar=True),
        # the rows of 64 decoding sequences with long histories, 16-bit logits
        adjust("adjust_64x128256_long", batch=64, width=1, vocab=VOCAB, dtype="bf16", history=8000, biases=0, grammar=False),
        # every node of 16 trees, each row with its own branch's tokens
        adjust("adjust_464x128256_trees", batch=16, width=29, vocab=VOCAB, dtype="fp32", history=2000, biases=20, grammar=True),
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

    op = rng.choice(["chunk", "chunk", "chunk", "chunk", "write", "adjust", "adjust"])
    if op == "write":
        model = rng.choice(["8b", "1b", "70b"])
        hd = HEADS[model][2]
        return dict(op="write", model=model, dtype=rng.choice(["bf16", "fp16"]),
                    tokens=log_int(1, 8191 if model != "70b" else 4500), start=log_int(1, 100000),
                    rot=rng.choice([hd, hd, hd // 2]), interleaved=rng.random() < 0.5, norm=rng.random() < 0.7)
    if op == "adjust":
        batch = log_int(1, 64)
        width = rng.choice([1, 1, log_int(2, 64)])
        width = min(width, max(1, 464 // batch))
        return dict(op="adjust", batch=batch, width=width, vocab=log_int(2048, VOCAB),
                    dtype=rng.choice(["fp32", "bf16", "fp16"]), history=log_int(1, 8000), biases=rng.choice([0, log_int(1, 300)]),
                    grammar=rng.random() < 0.5)
    model = rng.choice(["8b", "1b", "70b"])
    Hq, _, hd = HEADS[model]
    kind = rng.choice(["decode", "chunk", "mixed"])
    batch = log_int(1, 32) if kind == "decode" else log_int(1, 8) if kind == "chunk" else log_int(2, 16)
    longest = 1 if kind == "decode" else log_int(2, 8191 // batch)
    # no more keys than the 8-bit batch, and no more scores (padded to the longest) than the long document
    top = min(32000, 280000 // batch, int(4.0e9 / (Hq * batch * longest)) - longest)
    new = [longest if kind == "chunk" else 1] * batch
    if kind == "mixed":
        new = [longest if i == 0 else rng.choice([1, 1, rng.randint(1, longest)]) for i in range(batch)]
    if kind == "chunk":
        new = [longest] + [rng.randint(max(1, longest // 2), longest) for _ in range(batch - 1)]
    window = rng.choice([0, 0, log_int(100, 5000)])
    return dict(op="chunk", model=model, dtype=rng.choice(["bf16", "fp16"]), cache=rng.choice(["16", "16", "8"]),
                new=",".join(map(str, new)), ctx=",".join(str(log_int(1, max(2, top))) for _ in range(batch)),
                window=window, sinks=rng.choice([0, 4, 33]) if window else 0)


# ---- inputs -----------------------------------------------------------------
def _dev(a, dtype):
    return torch.tensor(np.asarray(a), dtype=dtype, device="cuda")


def _quantise(x):
    """e4m3 entries of the last dimension's rows and the exponent (biased by 127) of each row's power of two: the
    smallest under which no entry passes 448."""
    x = x.float()
    most = x.abs().amax(-1)
    m, e = torch.frexp(most)  # m in [0.5, 1): most / 2^e; 448 is 0.875 * 2^9
    e = torch.where(most > 0, e - 9 + (m > 0.875).int(), -127)
    e = e.clamp(-126, 127)
    codes = torch.ldexp(x, -e[..., None]).to(torch.float8_e4m3fn)
    return codes, (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu)


def _power(scale):
    """The powers of two that stored exponents stand for."""
    return torch.exp2(scale.view(torch.uint8).float() - 127.0)


def prepare(case, seed):
    rs = np.random.RandomState(seed % (1 << 31))
    g = torch.Generator(device="cuda").manual_seed(seed)
    op = case["op"]
    s = dict(op=op)
    if op == "adjust":
        return _prepare_adjust(case, rs, g, s)
    Hq, Hkv, hd = HEADS[case["model"]]
    dt = DTYPES[case["dtype"]]
    if op == "write":
        T = case["tokens"]
        n_pages = -(-T // PAGE) + 2
        order = torch.randperm(n_pages, generator=g, device="cuda")
        at = torch.arange(T, device="cuda")
        # channels of their own size, as keys have
        size = torch.exp(0.7 * torch.randn((Hq + 2 * Hkv) * hd, generator=g, device="cuda"))
        s.update(Hq=Hq, Hkv=Hkv, hd=hd, interleaved=case["interleaved"], rot=case["rot"], eps=1e-5,
                 qkv=(size * torch.randn((T, (Hq + 2 * Hkv) * hd), generator=g, device="cuda")).to(dt),
                 pos=(at + case["start"]).to(torch.int32), slots=order[at // PAGE] * PAGE + at % PAGE,
                 freq=_dev(THETA ** (-2.0 * np.arange(case["rot"] // 2) / case["rot"]), torch.float32))
        for name in ("q_gain", "k_gain"):
            s[name] = (1 + 0.2 * torch.randn(hd, generator=g, device="cuda")).to(dt) if case["norm"] else None
        for name in ("k", "v"):
            s[name + "_cache"] = torch.zeros((n_pages, Hkv, PAGE, hd), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
            s[name + "_scale"] = torch.ones((n_pages, Hkv, PAGE), dtype=torch.uint8, device="cuda").view(torch.float8_e8m0fnu)
        return s
    new, ctx = _ints(case["new"]), _ints(case["ctx"])
    need = [-(-(c + n) // PAGE) for c, n in zip(ctx, new)]
    order = rs.permutation(sum(need) + 3)
    table, at = np.zeros((len(new), max(need)), np.int64), 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    s.update(window=case["window"], sinks=case["sinks"], table=_dev(table, torch.int32), ctx=_dev(ctx, torch.int32),
             starts=_dev(np.cumsum([0] + new), torch.int32), longest=max(new))
    # scores with a spread of about 1.5, so that some keys stand out of a long context
    s["q"] = (1.5 * torch.randn((sum(new), Hq, hd), generator=g, device="cuda")).to(dt)
    for name in ("k", "v"):
        x = torch.randn((len(order), Hkv, PAGE, hd), generator=g, device="cuda")
        s[name + "_scale"] = None
        if case["cache"] == "8":
            size = torch.exp(0.5 * torch.randn((len(order), Hkv, PAGE, 1), generator=g, device="cuda"))
            s[name + "_cache"], s[name + "_scale"] = _quantise(x * size if name == "v" else x)
        else:
            s[name + "_cache"] = x.to(dt)
    return s


def _prepare_adjust(case, rs, g, s):
    B, N, V, L = case["batch"], case["width"], case["vocab"], case["history"]
    R = B * N
    z = 2.0 * torch.randn((R, V), generator=g, device="cuda")
    hot = torch.randint(0, V, (R, 64), generator=g, device="cuda")
    s["logits"] = z.scatter_add(1, hot, 14.0 * torch.rand((R, 64), generator=g, device="cuda")).to(DTYPES[case["dtype"]])
    # words come back as they do in text: few often, most seldom
    often = lambda shape: np.minimum((np.exp(rs.uniform(0, math.log(V), shape)) * 7919).astype(np.int64) % V, V - 1)  # noqa: E731
    lens = rs.randint(max(1, L // 2), L + 1, B)
    s.update(history=_dev(often((B, L)), torch.int32), hist_len=_dev(lens, torch.int32),
             prompt_len=_dev((lens * rs.uniform(0.2, 0.8, B)).astype(np.int64), torch.int32),
             repetition=_dev(rs.uniform(1.0, 1.3, B), torch.float32), frequency=_dev(rs.uniform(0, 0.5, B), torch.float32),
             presence=_dev(rs.uniform(0, 0.5, B), torch.float32), bias_ids=None, bias=None, allowed=None, tokens=None, mask=None)
    if case["biases"]:
        ids = np.stack([rs.choice(V, case["biases"], replace=False) for _ in range(B)])
        s.update(bias_ids=_dev(ids, torch.int32), bias=_dev(rs.uniform(-5, 5, ids.shape), torch.float32))
    if case["grammar"]:  # half of the rows free, the others down to an eighth of the vocabulary
        W = -(-V // 32)
        words = torch.randint(-2 ** 31, 2 ** 31, (3, R, W), generator=g, device="cuda")
        words = words[0] & words[1] & words[2]
        free = torch.rand(R, generator=g, device="cuda") < 0.5
        s["allowed"] = torch.where(free[:, None], -1, words).to(torch.int32)
    if N > 1:
        parents = np.stack([[-1] + [rs.randint(max(0, i - 12), i) for i in range(1, N)] for _ in range(B)])
        words = np.zeros((B, N, -(-N // 64)), np.uint64)
        for i in range(N):
            if i:
                words[:, i] = words[np.arange(B), parents[:, i]]
            words[:, i, i // 64] |= np.uint64(1) << np.uint64(i % 64)
        s.update(tokens=_dev(often((B, N)), torch.int32), mask=_dev(words.view(np.int64), torch.int64))
    return s


# ---- one pass ---------------------------------------------------------------
def run(s):
    if own:
        from paper_2504_18583_gb300 import tree
        return _own(s, tree)
    return _PLAIN[s["op"]](s)


def _own(s, tree):
    op = s["op"]
    if op == "chunk":
        return tree.chunk_attention(s["q"], s["k_cache"], s["v_cache"], s["table"], s["starts"], s["ctx"], window=s["window"],
                                    sinks=s["sinks"], k_scale=s["k_scale"], v_scale=s["v_scale"])
    if op == "write":
        q = tree.qk_norm_rope(s["qkv"], s["Hq"], s["Hkv"], s["pos"], s["slots"], s["k_cache"], s["v_cache"], s["freq"],
                              q_gain=s["q_gain"], k_gain=s["k_gain"], eps=s["eps"], interleaved=s["interleaved"],
                              k_scale=s["k_scale"], v_scale=s["v_scale"])
        return q, s["k_cache"], s["k_scale"], s["v_cache"], s["v_scale"]
    return tree.adjust_logits(s["logits"], s["history"], s["hist_len"], prompt_len=s["prompt_len"], repetition=s["repetition"],
                              frequency=s["frequency"], presence=s["presence"], bias_ids=s["bias_ids"], bias=s["bias"],
                              allowed=s["allowed"], tokens=s["tokens"], mask=s["mask"])


def _keys(cache, scale, table):
    """[B, Hkv, P * 16, hd] in 32 bits of a paged cache."""
    x = cache.view(torch.uint8)[table.long()].view(cache.dtype).float() if scale is not None else cache[table.long()].float()
    if scale is not None:
        x = x * _power(scale)[table.long()][..., None]
    return x.permute(0, 2, 1, 3, 4).reshape(x.shape[0], x.shape[2], -1, x.shape[4])


def _plain_chunk(s):
    T, Hq, hd = s["q"].shape
    starts, ctx, N = s["starts"].long(), s["ctx"].long(), s["longest"]
    k, v = _keys(s["k_cache"], s["k_scale"], s["table"]), _keys(s["v_cache"], s["v_scale"], s["table"])
    B, Hkv, n_keys, _ = k.shape
    row = starts[:-1, None] + torch.arange(N, device="cuda")  # the batch padded to its longest chunk
    live = row < starts[1:, None]
    q = s["q"].float()[row.clamp(max=T - 1)].view(B, N, Hkv, -1, hd).permute(0, 2, 1, 3, 4).reshape(B, Hkv, -1, hd)
    score = (q @ k.transpose(2, 3)).mul_(hd ** -0.5).view(B, Hkv, N, -1, n_keys)
    pos = (ctx[:, None] + torch.arange(N, device="cuda"))[..., None]
    j = torch.arange(n_keys, device="cuda")
    sees = j <= pos
    if s["window"]:
        sees &= (j > pos - s["window"]) | (j < s["sinks"])
    score.masked_fill_(~sees[:, None, :, None], float("-inf"))
    w = score.sub_(score.amax(-1, keepdim=True)).exp_()
    total = w.sum(-1, keepdim=True)
    o = (w.view(B, Hkv, -1, n_keys) @ v).view(B, Hkv, N, -1, hd) / total
    return o.permute(0, 2, 1, 3, 4).reshape(B, N, Hq, hd)[live].to(s["q"].dtype)


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


def _plain_write(s):
    Hq, Hkv, hd, dt = s["Hq"], s["Hkv"], s["hd"], s["qkv"].dtype
    x = s["qkv"].float().view(-1, Hq + 2 * Hkv, hd)
    q, k, v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    # angles in 64 bits, so that a far position does not wear the frequency's bits away
    angle = (s["pos"].double()[:, None] * s["freq"].double()[None])[:, None]
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    if s["q_gain"] is not None:
        q = q * torch.rsqrt(q.square().mean(-1, keepdim=True) + s["eps"]) * s["q_gain"].float()
        k = k * torch.rsqrt(k.square().mean(-1, keepdim=True) + s["eps"]) * s["k_gain"].float()
    q = _rotate(q, cos, sin, s["rot"], s["interleaved"]).to(dt)
    k = _rotate(k, cos, sin, s["rot"], s["interleaved"])
    page, at = s["slots"] // PAGE, s["slots"] % PAGE
    for name, rows in (("k", k), ("v", v)):
        codes, scale = _quantise(rows)
        s[name + "_cache"].view(torch.uint8)[page, :, at] = codes.view(torch.uint8)
        s[name + "_scale"].view(torch.uint8)[page, :, at] = scale.view(torch.uint8)
    return q, s["k_cache"], s["k_scale"], s["v_cache"], s["v_scale"]


def _bits(words, n):
    """[..., n] truth of packed words, the lowest column in the lowest bit."""
    per = words.element_size() * 8
    x = (words[..., None] >> torch.arange(per, dtype=words.dtype, device=words.device)) & 1
    return (x == 1).flatten(-2)[..., :n]


def _plain_adjust(s):
    z = s["logits"].float()
    R, V = z.shape
    B, L = s["history"].shape
    N = R // B
    at = torch.arange(L, device="cuda")
    there = at < s["hist_len"][:, None]
    ids = s["history"].long()
    one = torch.zeros((B, V), dtype=torch.int32, device="cuda")
    count = one.scatter_add(1, ids, (there & (at >= s["prompt_len"][:, None])).int())[:, None].expand(B, N, V)
    seen = (one.scatter_add(1, ids, there.int()) > 0)[:, None].expand(B, N, V)
    if s["tokens"] is not None:
        path = _bits(s["mask"], N)
        own_ids = s["tokens"].long()[:, None].expand(B, N, N)
        count = count.scatter_add(2, own_ids, path.int())
        seen = seen | (count > 0)
    z = z.view(B, N, V)
    rep = s["repetition"][:, None, None]
    z = torch.where(seen, torch.where(z > 0, z / rep, z * rep), z)
    z = z - s["frequency"][:, None, None] * count - s["presence"][:, None, None] * (count > 0)
    if s["bias_ids"] is not None:
        z = z + torch.zeros((B, V), device="cuda").scatter_add(1, s["bias_ids"].long(), s["bias"])[:, None]
    z = z.view(R, V)
    if s["allowed"] is not None:
        z = torch.where(_bits(s["allowed"], V), z, float("-inf"))
    return z.to(s["logits"].dtype)


_PLAIN = {"chunk": _plain_chunk, "write": _plain_write, "adjust": _plain_adjust}


# ---- what a pass cannot do without -------------------------------------------
def work(case):
    op = case["op"]
    if op == "adjust":
        size = 4 if case["dtype"] == "fp32" else 2
        n = case["batch"] * case["width"] * case["vocab"]
        return dict(bytes=2 * n * size + (n // 8 if case["grammar"] else 0) + case["batch"] * (3 * case["history"] + 8 * case["biases"]),
                    flops=4 * n)
    Hq, Hkv, hd = HEADS[case["model"]]
    if op == "write":
        T = case["tokens"]
        n = T * (Hq + 2 * Hkv) * hd
        return dict(bytes=2 * n + 2 * T * Hq * hd + 2 * T * Hkv * (hd + 1) + 12 * T, flops=8 * n)
    token = Hkv * (2 * (hd + 1) if case["cache"] == "8" else 4 * hd)  # bytes of a key and a value
    window, sinks = case["window"], case["sinks"]
    keys = pairs = rows = 0
    for n, c in zip(_ints(case["new"]), _ints(case["ctx"])):
        first = max(0, c - window + 1) if window else 0  # the earliest key in the first row's window
        keys += c + n - first + min(first, sinks)
        p = np.arange(c, c + n, dtype=np.int64)
        low = np.maximum(0, p - window + 1) if window else np.zeros_like(p)
        pairs += int((p + 1 - low + np.minimum(low, sinks)).sum())
        rows += n
    return dict(bytes=keys * token + 4 * rows * Hq * hd, flops=4 * hd * Hq * pairs)


# ---- the operators' definitions in 64 bits -----------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    return {"chunk": _exact_chunk, "write": _exact_write, "adjust": _exact_adjust}[case["op"]](s)


def _values(cache, scale, pages):
    """[Hkv, tokens, hd] in 64 bits of a sequence's pages."""
    x = cache.view(torch.uint8)[pages].view(cache.dtype).double() if scale is not None else cache[pages].double()
    if scale is not None:
        x = torch.ldexp(x, scale.view(torch.uint8)[pages][..., None].int() - 127)
    return x.transpose(0, 1).reshape(cache.shape[1], -1, cache.shape[3])


def _exact_chunk(s):
    """Sequence by sequence, head by head, 512 rows at a time."""
    T, Hq, hd = s["q"].shape
    starts, ctx = s["starts"].tolist(), s["ctx"].tolist()
    if sum((starts[b + 1] - starts[b]) * (ctx[b] + starts[b + 1] - starts[b]) for b in range(len(ctx))) * Hq > 5e9:
        return None
    out = torch.empty((T, Hq, hd), dtype=torch.float64, device="cuda")
    for b, c in enumerate(ctx):
        n = starts[b + 1] - starts[b]
        pages = s["table"][b, :-(-(c + n) // PAGE)].long()
        K, V = _values(s["k_cache"], s["k_scale"], pages), _values(s["v_cache"], s["v_scale"], pages)
        share = Hq // K.shape[0]
        for r0 in range(0, n, 512):
            r1 = min(n, r0 + 512)
            age = torch.arange(c + r0, c + r1, device="cuda")[:, None] - torch.arange(c + r1, device="cuda")[None]
            hidden = age < 0
            if s["window"]:
                hidden |= (age >= s["window"]) & (torch.arange(c + r1, device="cuda")[None] >= s["sinks"])
            for h in range(Hq):
                a = s["q"][starts[b] + r0:starts[b] + r1, h].double() @ K[h // share, :c + r1].T / math.sqrt(hd)
                out[starts[b] + r0:starts[b] + r1, h] = torch.softmax(a.masked_fill_(hidden, -math.inf), -1) @ V[h // share, :c + r1]
    return out


def _exact_write(s):
    Hq, Hkv, hd, half = s["Hq"], s["Hkv"], s["hd"], s["rot"] // 2
    x = s["qkv"].cpu().double().numpy().reshape(-1, Hq + 2 * Hkv, hd)
    angle = s["pos"].cpu().double().numpy()[:, None] * s["freq"].cpu().double().numpy()[None]
    turn = np.exp(1j * angle)[:, None]
    heads = []
    for lo, hi, gain in ((0, Hq, s["q_gain"]), (Hq, Hq + Hkv, s["k_gain"])):
        y = x[:, lo:hi].copy()
        if gain is not None:
            y = y / np.sqrt(np.mean(y * y, -1, keepdims=True) + s["eps"]) * gain.cpu().double().numpy()
        a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if s["interleaved"] else (slice(0, half), slice(half, 2 * half))
        c = (y[..., a] + 1j * y[..., b]) * turn
        y[..., a], y[..., b] = c.real, c.imag
        heads.append(y)
    slots = s["slots"].cpu().numpy()
    out = [torch.from_numpy(heads[0])]
    for name, rows in (("k", heads[1]), ("v", x[:, Hq + Hkv:])):
        codes, scales = s[name + "_cache"].cpu().double().numpy(), np.exp2(s[name + "_scale"].cpu().view(torch.uint8).double().numpy() - 127)
        power = np.exp2(np.clip(np.ceil(np.log2(np.maximum(np.abs(rows).max(-1), 1e-300) / TOP8)), -126, 127))
        y = rows / power[..., None]
        step = np.exp2(np.maximum(np.floor(np.log2(np.maximum(np.abs(y), 1e-300))), -6) - 3)  # three bits behind the first
        codes[slots // PAGE, :, slots % PAGE] = np.round(y / step) * step
        scales[slots // PAGE, :, slots % PAGE] = power
        out += [torch.from_numpy(codes), torch.from_numpy(scales)]
    return tuple(out)


def _exact_adjust(s):
    z = s["logits"].double()
    R, V = z.shape
    B = s["history"].shape[0]
    N = R // B
    hist, hist_len, prompt_len = s["history"].cpu().numpy(), s["hist_len"].tolist(), s["prompt_len"].tolist()
    rep, freq, pres = (s[n].cpu().double().numpy() for n in ("repetition", "frequency", "presence"))
    out = z.cpu().numpy()
    for r in range(R):
        b, i = divmod(r, N)
        said = hist[b, prompt_len[b]:hist_len[b]]
        if s["tokens"] is not None:
            words = s["mask"][b, i].cpu().numpy().view(np.uint8)
            said = np.concatenate([said, s["tokens"][b].cpu().numpy()[np.unpackbits(words, bitorder="little")[:N].astype(bool)]])
        ids = np.unique(np.concatenate([hist[b, :hist_len[b]], said]))
        out[r, ids] = np.where(out[r, ids] > 0, out[r, ids] / rep[b], out[r, ids] * rep[b])
        ids, count = np.unique(said, return_counts=True)
        out[r, ids] -= freq[b] * count + pres[b]
        if s["bias_ids"] is not None:
            np.add.at(out[r], s["bias_ids"][b].cpu().numpy(), s["bias"][b].cpu().double().numpy())
        if s["allowed"] is not None:
            words = s["allowed"][r].cpu().numpy().view(np.uint8)
            out[r, np.unpackbits(words, bitorder="little")[:V] == 0] = -np.inf
    return torch.from_numpy(out)
