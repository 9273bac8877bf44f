"""The operators around a quantised cache, as cases that can be timed and compared: norms of queries and keys for each head with the
rotation to their positions (one axis or several) and the fill of a cache of pages in one pass, the cache held in 16, 8 or 4 bits; reading such
a cache back; attention over it; and attention of a tree of drafted tokens.

A case is a dict of plain values.  `prepare` makes what a program holds before the call, `run` is one pass: in elementary
torch operations, or, where `own` is true, through the public entry points.  `work` is what the pass cannot do without,
`exact` the result in 64 bits.

A quantised cache holds, for every token and kv head, 128 codes and a scale for every 32 of them: a byte b that stands for 2^(b - 127).  The codes are 8
bits (fp8: sign, 4 exponent bits, 3 mantissa bits, up to 448) or 4 bits (fp4: 0, 0.5, 1, 1.5, 2, 3, 4, 6 with a sign, channel 2i in the lower half of byte
i).  The scale is the smallest power of two (2^-126 at least) by which the block's largest magnitude is divided into the codes' range; codes are
rounded to nearest, ties to even.  A million tokens of keys and values of one layer are 4.1 GB in 16 bits, 2.1 in 8, 1.1 in 4.

Heads (query/kv) are those of the recall's workloads: 32/8, 28/4, 64/8, 16/4, 8/2; head dimension 128.
"""
import math

import torch

own = False  # set from outside: False computes the plain forms, True calls the framework

D = 128
HEADS = ((32, 8), (32, 8), (28, 4), (64, 8), (16, 4), (8, 2))
FLOATS = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-6
BASE = 500000.0
# 48 requests in the middle of their answers, from a first token to a document of 16K
BATCH_48 = ("1,2,31,32,33,64,65,127,128,129,255,300,411,512,513,640,777,900,1000,1023,1024,1025,1280,1500,1777,2000,2047,2049,2500,3000,"
            "3333,3500,4000,4097,4500,5000,5555,6000,6500,7000,7777,8192,9001,10000,11111,12000,14000,16384")


def listed():
    return [
        # Eight requests answer: one new token each, normed, turned, stored in 8 bits and read back. Nothing but latency.
        {"name": "fill_step_8", "kind": "fill", "q": "1,1,1,1,1,1,1,1", "kv": "1,17,900,2048,4097,5000,8191,9001", "Hq": 32, "Hkv": 8, "page": 16,
         "layout": "head", "dtype": "bf16", "format": "fp8", "norm": "both", "pairing": "half", "rotary": 128, "axes": 1},
        # A chunk of a streamed context with images in it: positions in time, height and width; norms; a cache in 16 bits.
        {"name": "fill_image_chunk", "kind": "fill", "q": "1028", "kv": "9220", "Hq": 32, "Hkv": 8, "page": 64, "layout": "head", "dtype": "bf16",
         "format": "plain", "norm": "both", "pairing": "half", "rotary": 128, "axes": 3},
        # Two chunks of a model kept in fp32 that turns half of each head, neighbours as pairs, into a cache of 4 bits. Ragged sizes.
        {"name": "fill_partial_f32", "kind": "fill", "q": "777,301", "kv": "1900,301", "Hq": 16, "Hkv": 4, "page": 32, "layout": "token", "dtype": "f32",
         "format": "fp4", "norm": "both", "pairing": "interleaved", "rotary": 64, "axes": 1},
        # A whole document at once, groups of seven heads, into a cache of 8 bits.
        {"name": "fill_prompt_64k", "kind": "fill", "q": "65539", "kv": "65539", "Hq": 28, "Hkv": 4, "page": 256, "layout": "head", "dtype": "bf16",
         "format": "fp8", "norm": "both", "pairing": "half", "rotary": 128, "axes": 1},
        # After a recall: keys and values of the 4100 tokens that were kept, out of a context of 128K.
        {"name": "read_kept", "kind": "read", "kv": "131072", "rows": "4100", "pick": "some", "what": "both", "Hkv": 8, "page": 64, "layout": "head",
         "dtype": "bf16", "format": "fp8", "to": "token"},
        # Before a recall: all keys of a million tokens, as the recall's key cache.
        {"name": "read_keys_1m", "kind": "read", "kv": "1000003", "rows": "1000003", "pick": "all", "what": "keys", "Hkv": 8, "page": 64, "layout": "head",
         "dtype": "bf16", "format": "fp8", "to": "head"},
        # One request, one token, the compressed prompt of a budget of 4096: the smallest call.
        {"name": "step_4k_fp8", "kind": "paged", "q": "1", "kv": "4097", "Hq": 32, "Hkv": 8, "page": 16, "layout": "head", "dtype": "bf16", "format": "fp8",
         "causal": True, "sink": 0, "window": 0},
        # A batch of requests with contexts of very different lengths.
        {"name": "step_batch_48_fp8", "kind": "paged", "q": ",".join(["1"] * 48), "kv": BATCH_48, "Hq": 28, "Hkv": 4, "page": 64, "layout": "token",
         "dtype": "bf16", "format": "fp8", "causal": True, "sink": 0, "window": 0},
        # One token over the uncompressed cache of a million tokens, in 4 bits.
        {"name": "step_1m_fp4", "kind": "paged", "q": "1", "kv": "1000003", "Hq": 32, "Hkv": 8, "page": 64, "layout": "head", "dtype": "bf16",
         "format": "fp4", "causal": True, "sink": 0, "window": 0},
        # A chunk that attends to all of a 64K context.
        {"name": "chunk_64k_fp8", "kind": "paged", "q": "1024", "kv": "66560", "Hq": 32, "Hkv": 8, "page": 64, "layout": "head", "dtype": "bf16",
         "format": "fp8", "causal": True, "sink": 0, "window": 0},
        # Four requests with eight drafted tokens each, contexts of different lengths; one has nothing but its draft.
        {"name": "tree_8", "kind": "tree", "q": "8,8,7,8", "kv": "4105,9009,7,300", "Hq": 32, "Hkv": 8, "page": 64, "layout": "head", "dtype": "bf16",
         "format": "plain", "padded": False},
        # Two requests with 64 and 61 drafted tokens over long contexts, in 8 bits.
        {"name": "tree_64_fp8", "kind": "tree", "q": "64,61", "kv": "131136,30061", "Hq": 32, "Hkv": 8, "page": 64, "layout": "head", "dtype": "bf16",
         "format": "fp8", "padded": True},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("fill", "fill", "read", "paged", "paged", "paged", "tree", "tree"))
    heads = rng.choice(HEADS)
    case = {"kind": kind, "Hq": heads[0], "Hkv": heads[1], "dtype": rng.choice(("bf16", "bf16", "bf16", "f32")), "page": rng.choice((16, 32, 64, 256)),
            "layout": rng.choice(("head", "token")), "format": rng.choice(("fp8", "fp8", "fp4"))}
    slow = 8 if case["dtype"] == "f32" else 1
    if kind == "fill":
        shape = rng.choice(("step", "chunk", "whole"))
        if shape == "step":
            n = _log(rng, 1, 128)
            q, kv = [1] * n, [_log(rng, 1, 9000) for _ in range(n)]
        elif shape == "chunk":
            q = [_log(rng, 2, 2048) for _ in range(rng.choice((1, 1, 2, 5)))]
            kv = [a + rng.choice((0, _log(rng, 1, 9000))) for a in q]
        else:
            q = kv = [_log(rng, 1000, 65536 // slow)]
        case.update(format=rng.choice(("plain", "fp8", "fp4")), norm=rng.choice(("both", "both", "none", "offset")), pairing=rng.choice(("half", "half", "interleaved")),
                    rotary=rng.choice((128, 128, 64, 32, 96)), axes=rng.choice((1, 1, 3)))
    elif kind == "read":
        del case["Hq"]
        n = rng.choice((1, 1, 3, 8))
        kv = [_log(rng, 1, 300000 // n // slow) for _ in range(n)]
        pick = rng.choice(("all", "some"))
        rows = kv if pick == "all" else [_log(rng, 1, 8192) for _ in kv]
        case.update(pick=pick, rows=",".join(map(str, rows)), what=rng.choice(("both", "keys")), to=rng.choice(("token", "head")), kv=",".join(map(str, kv)))
        return case
    elif kind == "paged":
        shape = rng.choice(("step", "steps", "few", "chunk", "stream"))
        if shape == "step":
            q, kv = [1], [_log(rng, 1, 1000000 // slow)]
        elif shape == "steps":
            n = _log(rng, 2, 96)
            q, kv = [1] * n, [_log(rng, 1, 16384 // (1 if n < 32 else 2)) for _ in range(n)]
        elif shape == "few":  # a question, or a few drafted tokens, to contexts already there; a request with nothing yet
            n = rng.choice((1, 3, 8))
            q = [_log(rng, 1, 64) for _ in range(n)]
            kv = [a + rng.choice((0, _log(rng, 1, 30000 // slow))) for a in q]
            if n == 3:
                q[1] = kv[1] = 0
        elif shape == "chunk":
            q = [_log(rng, 64, 1024 // (1 if case["Hq"] < 64 else 2))]
            kv = [q[0] + _log(rng, 1, 65536 // slow)]
        else:
            q = [_log(rng, 64, 1028) for _ in range(rng.choice((1, 1, 4)))]
            kv = [a + _log(rng, 1, 9000) for a in q]
        stream = shape == "stream"
        case.update(causal=stream or rng.random() < 0.85, sink=rng.choice((0, 4, 4)) if stream else 0, window=rng.choice((512, 512, 100, 1024)) if stream else 0)
        if not case["causal"]:
            case["sink"] = case["window"] = 0
    else:
        n = rng.choice((1, 2, 4, 8))
        q = [_log(rng, 1, 100) for _ in range(n)]
        kv = [a + rng.choice((0, _log(rng, 1, 60000 // n // slow), _log(rng, 1, 60000 // n // slow))) for a in q]
        case.update(format=rng.choice(("plain", "plain", "fp8", "fp4")), padded=rng.random() < 0.5)
    case["q"], case["kv"] = ",".join(map(str, q)), ",".join(map(str, kv))
    return case


def _ints(text):
    return [int(x) for x in text.split(",")]


def _starts(lens):
    at = [0]
    for n in lens:
        at.append(at[-1] + n)
    return torch.tensor(at, dtype=torch.int32, device="cuda")


# ---------------------------------------------------------------- the formats of a quantised cache

TOP = {"fp8": 1.75, "fp4": 1.5}        # the largest code's fraction
TOP_EXP = {"fp8": 8, "fp4": 2}         # and its exponent
LEAST_EXP = {"fp8": -6, "fp4": 0}      # the exponent below which codes lie evenly
FRACTION = {"fp8": 3, "fp4": 1}        # bits
FP4 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _times_two_to(x, e):
    """x * 2^e in 64 bits, e whole: a power of two from its bits (a pow or exp2 may be off by its last bit, and then halfway cases fall anywhere)."""
    return x.double() * ((e.long() + 1023) << 52).view(torch.float64)


def _quantised(x, fmt):
    """(values of the codes, exponents of the scales [..., 4]) of x [..., 128], in 64 bits: what lies next to a border has to fall on its side of it."""
    x = x.double().unflatten(-1, (D // 32, 32))
    fraction, power = torch.frexp(x.abs().amax(-1))  # in [0.5, 1)
    e = torch.where(fraction == 0, -126, power - 1 - TOP_EXP[fmt] + (2 * fraction > TOP[fmt]).int()).clamp_(min=-126)
    t = _times_two_to(x, -e[..., None])
    step = (torch.frexp(t)[1] - 1).clamp_(min=LEAST_EXP[fmt]) - FRACTION[fmt]
    return _times_two_to(torch.round(_times_two_to(t, -step)), step).flatten(-2), e


def _codes(x, fmt):
    """What a cache holds for x [..., 128]: codes (fp8: float8_e4m3fn [..., 128], fp4: uint8 [..., 64]) and scales uint8 [..., 4]."""
    c, e = _quantised(x, fmt)
    if fmt == "fp8":
        return c.float().to(torch.float8_e4m3fn), (e + 127).to(torch.uint8)
    table = torch.tensor(FP4, dtype=torch.float64, device=x.device)
    code = torch.searchsorted(table, c.abs()).to(torch.uint8) | (torch.signbit(c).to(torch.uint8) << 3)
    return code[..., 0::2] | (code[..., 1::2] << 4), (e + 127).to(torch.uint8)


def _values(codes, scales, fmt):
    """The numbers that codes and scales stand for, in 32 bits."""
    if fmt == "plain":
        return codes.float()
    if fmt == "fp8":
        x = codes.float()
    else:
        table = torch.tensor(FP4 + tuple(-v for v in FP4), dtype=torch.float32, device=codes.device)
        x = table[torch.stack((codes & 15, codes >> 4), -1).flatten(-2).int()]
    return (x.unflatten(-1, (D // 32, 32)) * (scales.int() << 23).view(torch.float32)[..., None]).flatten(-2)  # (a byte as the exponent of a float)


def _row_bytes(case):
    """Bytes of a token's 128 channels of one kv head in the cache."""
    return {"plain": D * (2 if case["dtype"] == "bf16" else 4), "fp8": D + 4, "fp4": D // 2 + 4}[case["format"]]


# ---------------------------------------------------------------- inputs

def _pool(case, kv, g):
    """Pages of a cache in no order, a few of them nobody's, zeros everywhere: {k_pages, v_pages [n, Hkv, page, .], scales of the same layout, table}."""
    P, Hkv, fmt = case["page"], case["Hkv"], case["format"]
    need = [-(-n // P) for n in kv]
    total = sum(need) + 3

    def pages(width, dtype):
        x = torch.zeros((total, P, Hkv, width) if case["layout"] == "token" else (total, Hkv, P, width), dtype=dtype, device="cuda")
        return x.permute(0, 2, 1, 3) if case["layout"] == "token" else x

    kind, width = {"plain": (FLOATS[case["dtype"]], D), "fp8": (torch.uint8, D), "fp4": (torch.uint8, D // 2)}[fmt]
    st = {name: pages(width, kind) for name in ("k_pages", "v_pages")}
    if fmt != "plain":
        st.update({name: pages(D // 32, torch.uint8) for name in ("k_scales", "v_scales")})
    if fmt == "fp8":
        st["k_pages"], st["v_pages"] = (st[n].view(torch.float8_e4m3fn) for n in ("k_pages", "v_pages"))
    order = torch.randperm(total, generator=g, device="cuda").to(torch.int32)
    table = torch.zeros(len(kv), max(max(need), 1), dtype=torch.int32, device="cuda")
    at = 0
    for s, n in enumerate(need):
        table[s, :n] = order[at:at + n]
        at += n
    st["table"] = table
    return st


def _bytes(x):
    return x.view(torch.uint8) if x.dtype == torch.float8_e4m3fn else x


def _into_pool(st, case, s, k, v):
    """Sequence s's keys and values [tokens, Hkv, 128] to its pages, some tokens at a time."""
    P, fmt = case["page"], case["format"]
    for a in range(0, k.shape[0], 1 << 17):
        for name, x in (("k", k[a:a + (1 << 17)]), ("v", v[a:a + (1 << 17)])):
            at = torch.arange(a, a + x.shape[0], device="cuda")
            page = st["table"][s][at // P].long()
            if fmt == "plain":
                st[name + "_pages"][page, :, at % P] = x
            else:
                codes, scales = _codes(x, fmt)
                _bytes(st[name + "_pages"])[page, :, at % P] = _bytes(codes)
                st[name + "_scales"][page, :, at % P] = scales


def _normal(g, *shape):
    return torch.randn(*shape, device="cuda", generator=g)


def _states(case, q, kv, g):
    """Queries [T, Hq, d], and the keys and values [tokens, Hkv, d] of every sequence: as in the recall's workloads the queries of a kv
    group share a direction and the channels a scale in U(0.5, 2); the first four tokens of a sequence draw much of the weight."""
    Hq, Hkv, dt = case["Hq"], case["Hkv"], FLOATS[case["dtype"]]
    common, sigma = _normal(g, Hkv, D), 0.5 + 1.5 * torch.rand(Hkv, D, device="cuda", generator=g)
    mean, spread = 0.3 * _normal(g, Hkv, D), 0.5 + torch.rand(Hkv, D, device="cuda", generator=g)
    qs = ((math.sqrt(0.75) * _normal(g, sum(q), Hkv, Hq // Hkv, D) + 0.5 * common[:, None]) * sigma[:, None]).reshape(sum(q), Hq, D).to(dt)
    drawn = 0.5 * common * sigma * 1.5
    for n in kv:
        k = _normal(g, n, Hkv, D) * sigma
        k[:4] += drawn
        yield qs, k.to(dt), (_normal(g, n, Hkv, D) * spread + mean).to(dt)


def _tree(case, seed):
    """Which of its sequence's drafted tokens each drafted token sees, itself and its ancestors, as bits of 32-bit words [T, words].  Where the trees are
    padded, a sequence's last two tokens (of three or more) are nobody's and see none."""
    import random

    rng, rows = random.Random(seed), []
    q = _ints(case["q"])
    words = max(1, -(-max(q) // 32))
    for n in q:
        seen = []
        for i in range(n):
            parent = rng.randrange(max(0, i - 12), i) if i else -1
            seen.append((seen[parent] if i else 0) | 1 << i)
        if case["padded"] and n > 2:
            seen[-2:] = 0, 0
        rows += seen
    flat = [(r >> (32 * w)) & 0xFFFFFFFF for r in rows for w in range(words)]
    return torch.tensor([x - (1 << 32) if x >> 31 else x for x in flat], dtype=torch.int32, device="cuda").reshape(len(rows), words)


def _frequencies(case):
    return [BASE ** (-2.0 * j / case["rotary"]) for j in range(case["rotary"] // 2)]


def _axes(case):
    """The axis that each rotary pair turns by: a quarter of them by time, then height and width in turn."""
    n = case["rotary"] // 2
    return [0] * n if case["axes"] == 1 else [0 if j < n // 4 else 1 + j % 2 for j in range(n)]


def _inputs(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    kv, Hkv, dt = _ints(case["kv"]), case["Hkv"], FLOATS[case["dtype"]]
    st = {"case": case, "kv_len": torch.tensor(kv, dtype=torch.int32, device="cuda"), "max_kv": max(kv), "total_kv": sum(kv)}
    st.update(_pool(case, kv, g))
    if case["kind"] == "read":
        for s, (_, k, v) in enumerate(_states(dict(case, Hq=Hkv), [0], kv, g)):
            _into_pool(st, case, s, k, v)
        rows = _ints(case["rows"])
        st["cu_q"] = _starts(rows)
        if case["pick"] == "some":  # ascending, as a recall leaves them
            st["tokens"] = torch.cat([(torch.rand(n, device="cuda", generator=g) * m).to(torch.int32).clamp_(max=m - 1).sort()[0] for n, m in zip(rows, kv)])
        return st
    q, Hq = _ints(case["q"]), case["Hq"]
    T = sum(q)
    st.update(cu_q=_starts(q), max_q=max(q))
    if case["kind"] == "fill":
        # what a fused projection leaves behind: a token's queries, keys and values in one row
        fused = _normal(g, T, (Hq + 2 * Hkv) * D).to(dt).reshape(T, Hq + 2 * Hkv, D)
        st["q"], st["k"], st["v"] = fused[:, :Hq], fused[:, Hq:Hq + Hkv], fused[:, Hq + Hkv:]
        st["inv_freq"] = torch.tensor(_frequencies(case), dtype=torch.float64, device="cuda")
        st["axis"] = torch.tensor(_axes(case), dtype=torch.int64, device="cuda")
        place = torch.cat([torch.arange(n - a, n, device="cuda") for a, n in zip(q, kv)]).to(torch.int32)
        # an image of 32 x 24 patches after every 1000 tokens: its patches share a time
        st["positions"] = place[None] if case["axes"] == 1 else torch.stack((place - place % 768, place // 24 % 32 + place // 768, place % 24 + place // 768)).to(torch.int32)
        for name in ("q_weight", "k_weight"):
            st[name] = (0.3 * _normal(g, D) + (0 if case["norm"] == "offset" else 1)).to(dt)
    else:
        for s, (qs, k, v) in enumerate(_states(case, q, kv, g)):
            st["q"] = qs
            _into_pool(st, case, s, k, v)
        if case["kind"] == "tree":
            st["tree"] = _tree(case, seed)
    return st


def prepare(case, seed):
    st = _inputs(case, seed)
    if own:
        _handles(st)
    return st


def _handles(st):
    """What a serving program keeps between calls beside its tensors: the cache's description, the frequency table, the norms' weights, the
    workspace, the output buffers."""
    import paper_2508_17892_amd as il

    case, dt = st["case"], FLOATS[st["case"]["dtype"]]
    if case["format"] == "plain":
        st["cache"] = il.PagedKV(st["k_pages"], st["v_pages"], st["table"], st["kv_len"], st["cu_q"])
    else:
        st["cache"] = il.QuantKV(st["k_pages"], st["v_pages"], st["k_scales"], st["v_scales"], st["table"], st["kv_len"], st["cu_q"])
    T, Hkv = int(st["cu_q"][-1]), case["Hkv"]

    def rows():
        if case.get("to") == "head":  # the recall's key cache
            return torch.empty(Hkv, T, D, dtype=dt, device="cuda").transpose(0, 1)
        return torch.empty(T, Hkv, D, dtype=dt, device="cuda")

    if case["kind"] == "fill":
        st["freqs"] = il.ilre_rope_frequencies(case["rotary"], BASE)
        st["pairing"] = il.ILRE_ROPE_HALF if case["pairing"] == "half" else il.ILRE_ROPE_INTERLEAVED
        st["norms"] = None if case["norm"] == "none" else il.HeadNorms(st["q_weight"], st["k_weight"], eps=EPS, offset=1.0 if case["norm"] == "offset" else 0.0)
        st["axes"] = None if case["axes"] == 1 else tuple(_axes(case))
        st["out"] = torch.empty(st["q"].shape, dtype=dt, device="cuda")
        st["k_out"], st["v_out"] = rows(), rows()
    elif case["kind"] == "read":
        st["k_out"], st["v_out"] = rows(), rows() if case["what"] == "both" else None
    else:
        st["out"] = torch.empty_like(st["q"])
        st["lse"] = torch.empty(st["q"].shape[:2], dtype=torch.float32, device="cuda")
        st["workspace"] = il.alloc_workspace_attention(T, len(st["kv_len"]), case["Hq"], Hkv, D, st["max_q"], st["max_kv"],
                                                       total_kv=st["total_kv"], dtype=il.ILRE_BF16 if case["dtype"] == "bf16" else il.ILRE_F32)


def _run_own(st):
    import paper_2508_17892_amd as il

    case = st["case"]
    if case["kind"] == "fill":
        q = il.ilre_norm_rope_append(st["q"], st["k"], st["v"], st["cache"], st["freqs"], None if case["axes"] == 1 else st["positions"], norms=st["norms"],
                                     axes=st["axes"], pairing=st["pairing"], q_out=st["out"])
        if case["format"] == "plain":
            return q, st["k_pages"], st["v_pages"]
        return q, *il.ilre_cache_read(st["cache"], q.shape[0], k_out=st["k_out"], v_out=st["v_out"])
    if case["kind"] == "read":
        k, v = il.ilre_cache_read(st["cache"], st["k_out"].shape[0], st.get("tokens"), k_out=st["k_out"], v_out=st["v_out"])
        return (k, v) if case["what"] == "both" else k
    if case["kind"] == "tree":
        return il.ilre_tree_attention(st["q"], st["cache"], st["tree"], max_q=st["max_q"], max_kv=st["max_kv"], total_kv=st["total_kv"],
                                      workspace=st["workspace"], out=st["out"], lse=st["lse"])
    return il.ilre_paged_attention(st["q"], st["cache"], max_q=st["max_q"], max_kv=st["max_kv"], total_kv=st["total_kv"], causal=case["causal"],
                                   sink=case["sink"], window=case["window"], workspace=st["workspace"], out=st["out"], lse=st["lse"])


# ---------------------------------------------------------------- plain forms

def _sequence_of(cu_q, T):
    """Of every new token: its sequence, and how many of the sequence's new tokens come before it."""
    t = torch.arange(T, device="cuda", dtype=torch.int32)
    seq = torch.searchsorted(cu_q, t, right=True) - 1
    return seq, t - cu_q[seq]


def _normed(x, weight, case):
    if case["norm"] == "none":
        return x
    w = weight.to(x.dtype) + (1 if case["norm"] == "offset" else 0)
    return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w


def _turn(x, cos, sin, case):
    """The first `rotary` channels of every head, pair by pair; the others as they are."""
    r = case["rotary"]
    head, rest = x[..., :r], x[..., r:]
    a, b = (head[..., :r // 2], head[..., r // 2:]) if case["pairing"] == "half" else (head[..., 0::2], head[..., 1::2])
    ta, tb = a * cos - b * sin, b * cos + a * sin
    turned = torch.cat((ta, tb), -1) if case["pairing"] == "half" else torch.stack((ta, tb), -1).flatten(-2)
    return torch.cat((turned, rest), -1)


def _plain_fill(st):
    case, P, dt = st["case"], st["case"]["page"], st["q"].dtype
    angle = st["positions"].double()[st["axis"]].T * st["inv_freq"]
    cos, sin = angle.cos()[:, None], angle.sin()[:, None]
    q = _turn(_normed(st["q"].float(), st["q_weight"], case), cos.float(), sin.float(), case).to(dt)
    if case["format"] != "plain":
        k, v = _turn(_normed(st["k"].double(), st["k_weight"], case), cos, sin, case), st["v"]
        read = [_times_two_to(c.unflatten(-1, (D // 32, 32)), e[..., None]).flatten(-2).to(dt) for c, e in (_quantised(k, case["format"]), _quantised(v, case["format"]))]
        return q, read[0], read[1]
    k = _turn(_normed(st["k"].float(), st["k_weight"], case), cos.float(), sin.float(), case).to(dt)
    seq, i = _sequence_of(st["cu_q"], q.shape[0])
    at = st["kv_len"][seq] - (st["cu_q"][seq + 1] - st["cu_q"][seq]) + i
    page = st["table"][seq, (at // P).long()].long()
    st["k_pages"][page, :, (at % P).long()] = k
    st["v_pages"][page, :, (at % P).long()] = st["v"]
    return q, st["k_pages"], st["v_pages"]


def _plain_read(st):
    case, P, T = st["case"], st["case"]["page"], st["tokens"].shape[0] if "tokens" in st else st["total_kv"]
    seq, i = _sequence_of(st["cu_q"], T)
    at = st["tokens"] if "tokens" in st else i
    page, cell = st["table"][seq, (at // P).long()].long(), (at % P).long()

    def rows(name):
        return _values(_bytes(st[name + "_pages"])[page, :, cell].view(st[name + "_pages"].dtype), st[name + "_scales"][page, :, cell], case["format"]).to(FLOATS[case["dtype"]])

    return (rows("k"), rows("v")) if case["what"] == "both" else rows("k")


def _seen(st, S, Mq, Mk):
    """Which tokens each new one sees: bool [S, Mq, Mk]."""
    case, kv_len, cu = st["case"], st["kv_len"], st["cu_q"]
    q_len = cu[1:] - cu[:-1]
    t = torch.arange(Mk, device="cuda", dtype=torch.int32)[None, None]
    i = torch.arange(Mq, device="cuda", dtype=torch.int32)[None, :, None]
    before = (kv_len - q_len)[:, None, None]
    seen = (t < kv_len[:, None, None]).expand(S, Mq, Mk)
    if case["kind"] == "tree":
        at = (cu[:-1, None] + i[0, :, 0]).clamp_(max=st["q"].shape[0] - 1).long()
        words = st["tree"][at]  # [S, Mq, words]
        bit = torch.arange(words.shape[-1] * 32, device="cuda")
        bits = ((words[..., bit // 32] >> (bit % 32).int()) & 1).bool()
        j = (t - before).clamp(0, bits.shape[-1] - 1).expand(S, Mq, Mk).long()
        return seen & ((t < before) | bits.gather(2, j))
    place = before + i
    if case["causal"]:
        seen = seen & (t <= place)
    if case["window"]:
        seen = seen & ((t > place - case["window"]) | (t < case["sink"]))
    return seen


def _plain_attention(st):
    case, q = st["case"], st["q"]
    cu, T, S, Hkv, fmt = st["cu_q"], st["q"].shape[0], len(st["kv_len"]), st["case"]["Hkv"], st["case"]["format"]
    G, Mq, Mk = case["Hq"] // Hkv, st["max_q"], st["max_kv"]
    table = st["table"][:, :-(-max(Mk, 1) // case["page"])].long()

    def states(name):
        x, sc = st[name + "_pages"], st.get(name + "_scales")
        x = _values(_bytes(x)[table].view(x.dtype), None if sc is None else sc[table], fmt)
        return x.permute(0, 2, 1, 3, 4).reshape(S, Hkv, -1, D)[:, :, :Mk].contiguous()

    at = (cu[:-1, None] + torch.arange(Mq, device="cuda")).clamp_(max=T - 1).long()
    rows = (q[at].float() * (1 / math.sqrt(D))).reshape(S, Mq, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(S, Hkv, G * Mq, D)
    x = torch.matmul(rows, states("k").transpose(-1, -2)).reshape(S, Hkv, G, Mq, Mk)
    x.masked_fill_(~_seen(st, S, Mq, Mk)[:, None, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    top = torch.where(top.isinf(), torch.zeros_like(top), top)
    x.sub_(top).exp_()
    total = x.sum(-1, keepdim=True)
    out = torch.matmul(x.reshape(S, Hkv, G * Mq, Mk), states("v")).reshape(S, Hkv, G, Mq, D) / torch.where(total > 0, total, torch.ones_like(total))
    lse = (top + total.log())[..., 0]
    seq, i = _sequence_of(cu, T)
    return (out.permute(0, 3, 1, 2, 4).reshape(S, Mq, Hkv * G, D)[seq, i.long()].to(q.dtype), lse.permute(0, 3, 1, 2).reshape(S, Mq, Hkv * G)[seq, i.long()].contiguous())


def run(st):
    if own:
        return _run_own(st)
    kind = st["case"]["kind"]
    return _plain_fill(st) if kind == "fill" else _plain_read(st) if kind == "read" else _plain_attention(st)


# ---------------------------------------------------------------- what it takes, and the results in 64 bits

def _seen_by(case, q, kv):
    """(pairs of a row and a token it sees, tokens that any row sees) of one sequence."""
    if case["kind"] == "tree":  # about half of the drafted tokens' pairs at most; the context's are what counts
        return q * (kv - q) + q * (q + 1) // 2, kv
    if not case["causal"]:
        return q * kv, kv if q else 0
    pairs = 0
    for p in range(kv - q, kv):
        n = p + 1
        pairs += min(n, case["window"] + min(case["sink"], max(0, n - case["window"]))) if case["window"] else n
    first = kv - q + 1 - case["window"] if case["window"] else 0
    return pairs, kv - max(0, first) + min(case["sink"], max(0, first)) if q else 0


def work(case):
    es, Hkv, row = 2 if case["dtype"] == "bf16" else 4, case["Hkv"], _row_bytes(case)
    if case["kind"] == "read":
        n = sum(_ints(case["rows"])) * Hkv * (2 if case["what"] == "both" else 1)
        return {"bytes": n * (row + D * es), "flops": n * D}
    q, kv = _ints(case["q"]), _ints(case["kv"])
    T, Hq = sum(q), case["Hq"]
    if case["kind"] == "fill":  # states in, queries out, the cache's rows written; where they are quantised, the rows read back
        back = 0 if case["format"] == "plain" else 2 * T * Hkv * D * es
        return {"bytes": T * (2 * Hq + 2 * Hkv) * D * es + 2 * T * Hkv * row + back, "flops": T * (Hq + Hkv) * (3 * case["rotary"] + 4 * D)}
    seen = [_seen_by(case, a, b) for a, b in zip(q, kv)]
    return {"bytes": 2 * T * Hq * D * es + 2 * Hkv * sum(n for _, n in seen) * row + 4 * T * Hq + (_words(q) * 4 * T if case["kind"] == "tree" else 0),
            "flops": 4 * D * Hq * sum(p for p, _ in seen)}


def _words(q):
    return max(1, -(-max(q) // 32))


def _power(e):
    return torch.tensor([2.0 ** i for i in range(-200, 201)], dtype=torch.float64, device=e.device)[e.long() + 200]


def _exact_values(pages, scales, fmt):
    """Numbers of codes (as the cache holds them) in 64 bits, by the formats' definition bit by bit."""
    if fmt == "plain":
        return pages.double()
    c = _bytes(pages).long()
    if fmt == "fp4":
        c = torch.stack((c & 15, c >> 4), -1).flatten(-2)
        sign, exponent, fraction, bits, bias = c >> 3, (c >> 1) & 3, c & 1, 1, 1
    else:
        sign, exponent, fraction, bits, bias = c >> 7, (c >> 3) & 15, c & 7, 3, 7
    whole = torch.where(exponent > 0, (1 << bits) + fraction, fraction).double()
    x = whole * _power(exponent.clamp(min=1) - bias - bits) * (1 - 2 * sign).double()
    return x * _power(scales.long() - 127).repeat_interleave(32, -1)


def _exact_stored(x, fmt):
    """The numbers that a cache gives back for x [..., 128] (64 bits): the scale by trying powers of two, the code by looking for its neighbours in the list of all."""
    if fmt == "fp4":
        table = torch.tensor(FP4, dtype=torch.float64, device=x.device)
    else:
        table = torch.tensor([(m if e == 0 else 8 + m) * 2.0 ** (max(e, 1) - 10) for e in range(16) for m in range(8)][:-1], dtype=torch.float64, device=x.device)
    got = torch.empty_like(x)
    for a in range(0, x.shape[0], 8192):
        y = x[a:a + 8192].unflatten(-1, (D // 32, 32))
        top = y.abs().amax(-1, keepdim=True)
        scale = _power((torch.log2(top.clamp(min=1e-300)).floor() - TOP_EXP[fmt] - 2).clamp(min=-126.0))
        for _ in range(4):
            scale = torch.where(top > table[-1] * scale, 2 * scale, scale)
        t = y.abs() / scale
        above = torch.searchsorted(table, t.contiguous()).clamp(max=len(table) - 1)  # the first that is not below
        below = (above - 1).clamp(min=0)
        up, down = table[above] - t, t - table[below]
        code = torch.where((up < down) | ((up == down) & (above % 2 == 0)) | (up == 0), above, below)
        got[a:a + 8192] = (table[code] * torch.sign(y) * scale).flatten(-2)
    return got


def _exact_fill(case, st):
    half, r, T = case["pairing"] == "half", case["rotary"], st["q"].shape[0]
    freq = torch.tensor(_frequencies(case), dtype=torch.float64, device="cuda")
    place = torch.stack([st["positions"][a] for a in _axes(case)], 1).double()
    wheel = torch.polar(torch.ones_like(place), place * freq)[:, None]

    def ready(x, weight):
        x = x.double()
        if case["norm"] != "none":
            x = x / (x.square().sum(-1, keepdim=True) / D + EPS).sqrt() * (weight.double() + (1.0 if case["norm"] == "offset" else 0.0))
        head = x[..., :r]
        z = (torch.complex(head[..., :r // 2].contiguous(), head[..., r // 2:].contiguous()) if half else torch.view_as_complex(head.reshape(*head.shape[:-1], r // 2, 2).contiguous())) * wheel
        head = torch.cat((z.real, z.imag), -1) if half else torch.view_as_real(z).flatten(-2)
        return torch.cat((head, x[..., r:]), -1)

    q, k, v = ready(st["q"], st["q_weight"]), ready(st["k"], st["k_weight"]), st["v"].double()
    if case["format"] != "plain":
        return q, _exact_stored(k, case["format"]), _exact_stored(v, case["format"])
    kp, vp, P, row = st["k_pages"].double(), st["v_pages"].double(), case["page"], 0
    for s, (a, n) in enumerate(zip(_ints(case["q"]), _ints(case["kv"]))):
        at = torch.arange(n - a, n, device="cuda")
        page = st["table"][s][at // P].long()
        kp[page, :, at % P], vp[page, :, at % P] = k[row:row + a], v[row:row + a]
        row += a
    return q, kp, vp


def _exact_read(case, st):
    P, row, got = case["page"], 0, ([], [])
    for s, (n, m) in enumerate(zip(_ints(case["rows"]), _ints(case["kv"]))):
        at = st["tokens"][row:row + n].long() if case["pick"] == "some" else torch.arange(m, device="cuda")
        row += n
        for b in range(0, n, 1 << 17):
            part = at[b:b + (1 << 17)]
            page = st["table"][s][part // P].long()
            for name, to in zip(("k", "v"), got):
                to.append(_exact_values(_bytes(st[name + "_pages"])[page, :, part % P], st[name + "_scales"][page, :, part % P], case["format"]))
    return (torch.cat(got[0]), torch.cat(got[1])) if case["what"] == "both" else torch.cat(got[0])


def exact(case, seed):
    st = _inputs(case, seed)
    if case["kind"] == "fill":
        return _exact_fill(case, st)
    if case["kind"] == "read":
        return _exact_read(case, st)
    q, kv = _ints(case["q"]), _ints(case["kv"])
    Hkv, G, P, fmt = case["Hkv"], case["Hq"] // case["Hkv"], case["page"], case["format"]
    out = torch.zeros(sum(q), case["Hq"], D, dtype=torch.float64, device="cuda")
    lse = torch.full((sum(q), case["Hq"]), -math.inf, dtype=torch.float64, device="cuda")
    row = 0
    for s, (a, n) in enumerate(zip(q, kv)):
        if a and n:
            place = torch.arange(n - a, n, device="cuda")[:, None]
            t = torch.arange(n, device="cuda")[None]
            if case["kind"] == "tree":
                hidden = torch.zeros(a, n, dtype=torch.bool, device="cuda")
                words = [[x & 0xFFFFFFFF for x in r] for r in st["tree"][row:row + a].tolist()]
                hidden[:, n - a:] = torch.tensor([[not (w[j // 32] >> (j % 32)) & 1 for j in range(a)] for w in words], device="cuda")
            else:
                hidden = t > place if case["causal"] else torch.zeros(a, n, dtype=torch.bool, device="cuda")
                if case["window"]:
                    hidden |= (t <= place - case["window"]) & (t >= case["sink"])
            pages = st["table"][s, :-(-n // P)].long()
            for h in range(Hkv):
                kh, vh = (_exact_values(_bytes(st[x + "_pages"])[pages, h].view(st[x + "_pages"].dtype), None if fmt == "plain" else st[x + "_scales"][pages, h], fmt).reshape(-1, D)[:n]
                          for x in ("k", "v"))
                for j in range(h * G, (h + 1) * G):
                    logits = st["q"][row:row + a, j].double() @ kh.T.contiguous() / math.sqrt(D)
                    logits.masked_fill_(hidden, -math.inf)
                    lse[row:row + a, j] = torch.logsumexp(logits, 1)
                    ok = lse[row:row + a, j] > -math.inf
                    weights = logits.sub_(torch.where(ok, lse[row:row + a, j], 0.0)[:, None]).exp_()
                    out[row:row + a, j] = weights @ vh
        row += a
    return out, lse
