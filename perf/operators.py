"""The operators around a recall, as cases that can be timed and compared: rotary positions with the fill of a paged cache,
attention of new tokens over that cache, and causal attention over whole packed prompts.

A case is a dict of plain values.  `prepare` makes what a program holds before the call, `run` is one pass: in elementary
torch operations, or, where `own` is true, through the public entry points.  `work` is what the pass cannot do without,
`exact` the result in 64 bits.

A context is streamed through the layers below the retrieval layer in chunks of new tokens: their queries and keys are turned
to their positions, keys and values go to the cache, and the chunk attends to the cache's sink part and window.  The question
and the answer's tokens attend to all of a cache, and the prompts that recalls leave behind, of different lengths, are
attended to whole.  Heads (query/kv) are those of the recall's workloads: 32/8, 28/4, 64/8, 16/4, 8/2; head dimension 128.
"""
import math

import torch

own = False  # set from outside: False computes the plain forms, True calls the framework

D = 128
HEADS = ((32, 8), (32, 8), (28, 4), (64, 8), (16, 4), (8, 2))
FLOATS = {"bf16": torch.bfloat16, "f32": torch.float32}
# 48 requests in the middle of their answers, from a first token to a document of 16K
BATCH_48 = ("1,2,31,32,33,64,65,127,128,129,255,300,411,512,513,640,777,900,1000,1023,1024,1025,1280,1500,1777,2000,2047,2049,2500,3000,"
            "3333,3500,4000,4097,4500,5000,5555,6000,6500,7000,7777,8192,9001,10000,11111,12000,14000,16384")


def listed():
    return [
        # Eight requests answer: one new token each, turned and stored. Nothing but latency.
        {"name": "rope_step_8", "kind": "rope", "q": "1,1,1,1,1,1,1,1", "kv": "1,17,900,2048,4097,5000,8191,9001", "Hq": 32, "Hkv": 8, "page": 16,
         "layout": "head", "dtype": "bf16", "pairing": "half", "rotary": 128, "scaling": "bands", "shift": 0},
        # A chunk of a streamed context (the first one brings the sink part along: 1024 + 4 tokens).
        {"name": "rope_chunk_1k", "kind": "rope", "q": "1028", "kv": "9220", "Hq": 32, "Hkv": 8, "page": 64, "layout": "head", "dtype": "bf16",
         "pairing": "half", "rotary": 128, "scaling": "bands", "shift": 0},
        # Two chunks of a model kept in fp32 that turns half of each head, neighbours as pairs; positions run ahead of the cache,
        # part of which was dropped. Ragged sizes.
        {"name": "rope_partial_f32", "kind": "rope", "q": "777,301", "kv": "1900,301", "Hq": 16, "Hkv": 4, "page": 32, "layout": "token", "dtype": "f32",
         "pairing": "interleaved", "rotary": 64, "scaling": "linear", "shift": 100003},
        # A whole document at once, groups of seven heads, frequencies scaled by parts.
        {"name": "rope_prompt_64k", "kind": "rope", "q": "65539", "kv": "65539", "Hq": 28, "Hkv": 4, "page": 256, "layout": "head", "dtype": "bf16",
         "pairing": "half", "rotary": 128, "scaling": "parts", "shift": 0},
        # One request, one token, the compressed prompt of a budget of 4096: the smallest call.
        {"name": "step_4k", "kind": "paged", "q": "1", "kv": "4097", "Hq": 32, "Hkv": 8, "page": 16, "layout": "head", "dtype": "bf16", "causal": True,
         "sink": 0, "window": 0},
        # A batch of requests with contexts of very different lengths.
        {"name": "step_batch_48", "kind": "paged", "q": ",".join(["1"] * 48), "kv": BATCH_48, "Hq": 28, "Hkv": 4, "page": 64, "layout": "token",
         "dtype": "bf16", "causal": True, "sink": 0, "window": 0},
        # One token over the uncompressed cache of a million tokens.
        {"name": "step_1m", "kind": "paged", "q": "1", "kv": "1000003", "Hq": 32, "Hkv": 8, "page": 64, "layout": "head", "dtype": "bf16", "causal": True,
         "sink": 0, "window": 0},
        # A chunk of a streamed context: sink part of 4, window of 512.
        {"name": "stream_chunk", "kind": "paged", "q": "1024", "kv": "9220", "Hq": 32, "Hkv": 8, "page": 64, "layout": "head", "dtype": "bf16",
         "causal": True, "sink": 4, "window": 512},
        # A chunk that attends to all of a 64K context.
        {"name": "chunk_64k", "kind": "paged", "q": "1024", "kv": "66560", "Hq": 32, "Hkv": 8, "page": 64, "layout": "head", "dtype": "bf16",
         "causal": True, "sink": 0, "window": 0},
        # Compressed prompts of several requests, packed.
        {"name": "prompts_packed", "kind": "prompt", "q": "1,4096,700,2047,33,4130,129,1025", "Hq": 32, "Hkv": 8, "dtype": "bf16", "causal": True, "sink": 0,
         "window": 0},
        # Short prompts in fp32, as a validation runs them.
        {"name": "prompts_f32", "kind": "prompt", "q": "500,77,900", "Hq": 8, "Hkv": 2, "dtype": "f32", "causal": True, "sink": 0, "window": 0},
        # One long prompt, uncompressed.
        {"name": "prompt_16k", "kind": "prompt", "q": "16384", "Hq": 32, "Hkv": 8, "dtype": "bf16", "causal": True, "sink": 0, "window": 0},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("rope", "paged", "paged", "paged", "prompt", "prompt"))
    heads = rng.choice(HEADS)
    case = {"kind": kind, "Hq": heads[0], "Hkv": heads[1], "dtype": rng.choice(("bf16", "bf16", "bf16", "f32"))}
    slow = 8 if case["dtype"] == "f32" else 1
    if kind == "rope":
        shape = rng.choice(("step", "chunk", "whole"))
        if shape == "step":
            n = _log(rng, 1, 128)
            q, kv = [1] * n, [_log(rng, 1, 9000) for _ in range(n)]
        elif shape == "chunk":
            q = [_log(rng, 2, 2048) for _ in range(rng.choice((1, 1, 2, 5)))]
            kv = [a + rng.choice((0, _log(rng, 1, 9000))) for a in q]
        else:
            q = kv = [_log(rng, 1000, 65536 // slow)]
        case.update(page=rng.choice((16, 32, 64, 256)), layout=rng.choice(("head", "token")), pairing=rng.choice(("half", "half", "interleaved")),
                    rotary=rng.choice((128, 128, 64, 32, 96)), scaling=rng.choice(("plain", "linear", "bands", "parts")),
                    shift=rng.choice((0, 0, 1000003)))
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
            q = [_log(rng, 64, 1024)]
            kv = [q[0] + _log(rng, 1, 65536 // slow)]
        else:
            q = [_log(rng, 64, 1028) for _ in range(rng.choice((1, 1, 4)))]
            kv = [a + _log(rng, 1, 9000) for a in q]
        stream = shape == "stream"
        case.update(page=rng.choice((16, 32, 64, 256)), layout=rng.choice(("head", "token")), causal=stream or rng.random() < 0.85,
                    sink=rng.choice((0, 4, 4)) if stream else 0, window=rng.choice((512, 512, 100, 1024)) if stream else 0)
        if not case["causal"]:
            case["sink"] = case["window"] = 0
    else:
        n = rng.choice((1, 2, 5, 12))
        most = (16384 if n == 1 else 8192 if n == 2 else 4200 if n == 5 else 2048) // (64 // case["Hq"] if case["Hq"] > 32 else 1)
        most = most // 2 if case["Hq"] == 64 else most // 8 if slow > 1 else most
        q = [_log(rng, 1 if n > 1 else 200, most) for _ in range(n)]
        kv = q
        case.update(causal=rng.random() < 0.85, sink=0, window=0)
        if case["causal"] and rng.random() < 0.25:
            case.update(sink=4, window=512)
    case["q"] = ",".join(map(str, q))
    if kind != "prompt":
        case["kv"] = ",".join(map(str, kv))
    return case


def _ints(text):
    return [int(x) for x in text.split(",")]


def _lens(case):
    q = _ints(case["q"])
    return q, _ints(case["kv"]) if "kv" in case else q


def _starts(lens):
    at = [0]
    for n in lens:
        at.append(at[-1] + n)
    return torch.tensor(at, dtype=torch.int32, device="cuda")


SCALING = {"plain": {}, "linear": {"factor": 4.0}, "bands": {"factor": 8.0, "low": 1.0, "high": 4.0, "original": 8192},
           "parts": {"factor": 16.0, "low": 1.0, "high": 32.0, "original": 4096}}
BASE = {"plain": 10000.0, "linear": 10000.0, "bands": 500000.0, "parts": 10000.0}


def _frequencies(rotary, kind):
    """Radians a position for every rotary pair, and what the turned part is multiplied with."""
    base, s = BASE[kind], SCALING[kind]
    freq = [base ** (-2.0 * j / rotary) for j in range(rotary // 2)]
    if kind == "linear":
        return [f / s["factor"] for f in freq], 1.0
    if kind == "bands":  # by how many turns a pair makes over the original length
        def band(f):
            turns = s["original"] * f / (2 * math.pi)
            keep = min(1.0, max(0.0, (turns - s["low"]) / (s["high"] - s["low"])))
            return f * keep + f / s["factor"] * (1 - keep)
        return [band(f) for f in freq], 1.0
    if kind == "parts":  # a ramp over the pairs' numbers between those that make `high` and `low` turns
        def pair(turns):
            return rotary * math.log(s["original"] / (turns * 2 * math.pi)) / (2 * math.log(base))
        first, last = max(math.floor(pair(s["high"])), 0), min(math.ceil(pair(s["low"])), rotary - 1)
        ramp = [min(1.0, max(0.0, (j - first) / max(last - first, 1e-3))) for j in range(rotary // 2)]
        return [f * (1 - r) + f / s["factor"] * r for f, r in zip(freq, ramp)], 0.1 * math.log(s["factor"]) + 1
    return freq, 1.0


def _pool(case, kv, g, fill=None):
    """Pages of a cache in no order, a few of them nobody's: (pages [n, Hkv, page, d], table [sequences, pages a sequence])."""
    P, Hkv = case["page"], case["Hkv"]
    need = [-(-n // P) for n in kv]
    total = sum(need) + 3
    shape = (total, P, Hkv, D) if case["layout"] == "token" else (total, Hkv, P, D)
    pages = [torch.empty(shape, dtype=FLOATS[case["dtype"]], device="cuda") for _ in range(2)]
    pages = [p.permute(0, 2, 1, 3) if case["layout"] == "token" else p for p in pages]
    order = torch.randperm(total, generator=g, device="cuda").to(torch.int32)
    table = torch.zeros(len(kv), max(max(need), 1), dtype=torch.int32, device="cuda")
    at = 0
    for s, n in enumerate(need):
        table[s, :n] = order[at:at + n]
        at += n
    return pages[0], pages[1], table


def _states(case, q, kv, g):
    """Queries [T, Hq, d], and the keys and values [tokens, Hkv, d] of every sequence: as in the recall's workloads the queries of a kv
    group share a direction and the channels a scale in U(0.5, 2); the first four tokens of a sequence draw much of the weight."""
    Hq, Hkv, dt = case["Hq"], case["Hkv"], FLOATS[case["dtype"]]
    def normal(*shape):
        return torch.randn(*shape, device="cuda", generator=g)
    common, sigma = normal(Hkv, D), 0.5 + 1.5 * torch.rand(Hkv, D, device="cuda", generator=g)
    mean, spread = 0.3 * normal(Hkv, D), 0.5 + torch.rand(Hkv, D, device="cuda", generator=g)
    qs = ((math.sqrt(0.75) * normal(sum(q), Hkv, Hq // Hkv, D) + 0.5 * common[:, None]) * sigma[:, None]).reshape(sum(q), Hq, D).to(dt)
    drawn = 0.5 * common * sigma * 1.5
    for n in kv:
        k = normal(n, Hkv, D) * sigma
        k[:4] += drawn
        yield qs, k.to(dt), (normal(n, Hkv, D) * spread + mean).to(dt)


def _inputs(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    q, kv = _lens(case)
    Hq, Hkv, dt = case["Hq"], case["Hkv"], FLOATS[case["dtype"]]
    T = sum(q)
    st = {"case": case, "cu_q": _starts(q), "max_q": max(q), "max_kv": max(kv), "total_kv": sum(kv)}
    st["kv_len"] = torch.tensor(kv, dtype=torch.int32, device="cuda")
    if case["kind"] == "rope":
        # what a fused projection leaves behind: a token's queries, keys and values in one row
        fused = torch.randn(T, (Hq + 2 * Hkv) * D, device="cuda", generator=g).to(dt).reshape(T, Hq + 2 * Hkv, D)
        st["q"], st["k"], st["v"] = fused[:, :Hq], fused[:, Hq:Hq + Hkv], fused[:, Hq + Hkv:]
        st["k_pages"], st["v_pages"], st["table"] = _pool(case, kv, g)
        for p in (st["k_pages"], st["v_pages"]):
            p.copy_(torch.randn(p.shape, device="cuda", generator=g))
        st["inv_freq"], st["magnitude"] = _frequencies(case["rotary"], case["scaling"])
        st["inv_freq_dev"] = torch.tensor(st["inv_freq"], dtype=torch.float64, device="cuda")
        own_place = torch.cat([torch.arange(n - a, n, device="cuda") for a, n in zip(q, kv)])
        st["positions"] = (own_place + case["shift"]).to(torch.int32)
    elif case["kind"] == "paged":
        st["k_pages"], st["v_pages"], st["table"] = _pool(case, kv, g)
        P = case["page"]
        for p in (st["k_pages"], st["v_pages"]):
            p.zero_()  # pages nobody has written to yet
        for s, (qs, k, v) in enumerate(_states(case, q, kv, g)):
            st["q"] = qs
            at = torch.arange(kv[s], device="cuda")
            page = st["table"][s][at // P].long()
            st["k_pages"][page, :, at % P] = k
            st["v_pages"][page, :, at % P] = v
    else:
        parts = list(_states(case, q, kv, g))
        st["q"] = parts[0][0]
        st["k"], st["v"] = (torch.cat([p[i] for p in parts]) for i in (1, 2))
    return st


def prepare(case, seed):
    st = _inputs(case, seed)
    if own:
        _handles(st)
    return st


def _handles(st):
    """What a serving program keeps between calls beside its tensors: the cache's description, the frequency table, the workspace, the
    output buffers."""
    import paper_2508_17892_amd as il

    case, q = st["case"], st["q"]
    if case["kind"] != "prompt":
        st["cache"] = il.PagedKV(st["k_pages"], st["v_pages"], st["table"], st["kv_len"], st["cu_q"])
    if case["kind"] == "rope":
        s = SCALING[case["scaling"]]
        kind = {"plain": il.ILRE_ROPE_PLAIN, "linear": il.ILRE_ROPE_LINEAR, "bands": il.ILRE_ROPE_BANDS, "parts": il.ILRE_ROPE_PARTS}[case["scaling"]]
        st["freqs"] = il.ilre_rope_frequencies(case["rotary"], BASE[case["scaling"]], scaling=kind, factor=s.get("factor", 1.0), low=s.get("low", 1.0),
                                               high=s.get("high", 1.0), original_len=s.get("original", 0))
        st["pairing"] = il.ILRE_ROPE_HALF if case["pairing"] == "half" else il.ILRE_ROPE_INTERLEAVED
        st["out"] = torch.empty(q.shape, dtype=q.dtype, device="cuda")
    else:
        st["out"] = torch.empty_like(q)
        st["lse"] = torch.empty(q.shape[:2], dtype=torch.float32, device="cuda")
        st["workspace"] = il.alloc_workspace_attention(q.shape[0], len(st["kv_len"]), case["Hq"], case["Hkv"], D, st["max_q"], st["max_kv"],
                                                       total_kv=st["total_kv"], dtype=il.ILRE_BF16 if case["dtype"] == "bf16" else il.ILRE_F32)


def _run_own(st):
    import paper_2508_17892_amd as il

    case = st["case"]
    if case["kind"] == "rope":
        q = il.ilre_rope_append(st["q"], st["k"], st["v"], st["cache"], st["freqs"], st["positions"] if case["shift"] else None,
                                pairing=st["pairing"], q_out=st["out"])
        return q, st["k_pages"], st["v_pages"]
    if case["kind"] == "paged":
        return il.ilre_paged_attention(st["q"], st["cache"], max_q=st["max_q"], max_kv=st["max_kv"], total_kv=st["total_kv"], causal=case["causal"],
                                       sink=case["sink"], window=case["window"], workspace=st["workspace"], out=st["out"], lse=st["lse"])
    return il.ilre_prompt_attention(st["q"], st["k"], st["v"], st["cu_q"], max_q=st["max_q"], causal=case["causal"], sink=case["sink"],
                                    window=case["window"], workspace=st["workspace"], out=st["out"], lse=st["lse"])


def _turn(x, cos, sin, case):
    """The first `rotary` channels of every head, pair by pair; the others as they are."""
    r = case["rotary"]
    head, rest = x[..., :r].float(), x[..., r:]
    a, b = (head[..., :r // 2], head[..., r // 2:]) if case["pairing"] == "half" else (head[..., 0::2], head[..., 1::2])
    ta, tb = a * cos - b * sin, b * cos + a * sin
    turned = torch.cat((ta, tb), -1) if case["pairing"] == "half" else torch.stack((ta, tb), -1).flatten(-2)
    return torch.cat((turned.to(x.dtype), rest), -1)


def _sequence_of(cu_q, T):
    """Of every new token: its sequence, and how many of the sequence's new tokens come before it."""
    t = torch.arange(T, device="cuda", dtype=torch.int32)
    seq = torch.searchsorted(cu_q, t, right=True) - 1
    return seq, t - cu_q[seq]


def _plain_rope(st):
    case, P = st["case"], st["case"]["page"]
    angle = st["positions"].double()[:, None] * st["inv_freq_dev"]
    cos = (angle.cos() * st["magnitude"]).float()[:, None]
    sin = (angle.sin() * st["magnitude"]).float()[:, None]
    seq, i = _sequence_of(st["cu_q"], st["q"].shape[0])
    at = st["kv_len"][seq] - (st["cu_q"][seq + 1] - st["cu_q"][seq]) + i
    page = st["table"][seq, (at // P).long()].long()
    st["k_pages"][page, :, (at % P).long()] = _turn(st["k"], cos, sin, case)
    st["v_pages"][page, :, (at % P).long()] = st["v"]
    return _turn(st["q"], cos, sin, case), st["k_pages"], st["v_pages"]


def _softmax_attention(q, k, v, q_len, kv_len, case):
    """Padded attention in 32 bits. q [S, Mq, Hq, d], k and v [S, Hkv, Mk, d] -> out [S, Mq, Hq, d], log of the rows' sums [S, Mq, Hq]."""
    S, Mq, Hq, _ = q.shape
    Hkv, Mk = k.shape[1], k.shape[2]
    G = Hq // Hkv
    q = (q.float() * (1 / math.sqrt(D))).reshape(S, Mq, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(S, Hkv, G * Mq, D)
    x = torch.matmul(q, k.transpose(-1, -2)).reshape(S, Hkv, G, Mq, Mk)
    t = torch.arange(Mk, device="cuda", dtype=torch.int32)[None, None]
    place = (kv_len - q_len)[:, None, None] + torch.arange(Mq, device="cuda", dtype=torch.int32)[None, :, None]
    seen = (t < kv_len[:, None, None]).expand(S, Mq, Mk)
    if case["causal"]:
        seen = seen & (t <= place)
    if case["window"]:
        seen = seen & ((t > place - case["window"]) | (t < case["sink"]))
    x.masked_fill_(~seen[:, None, None], -math.inf)
    top = x.amax(-1, keepdim=True) if Mk else x.new_full((S, Hkv, G, Mq, 1), -math.inf)
    top = torch.where(top.isinf(), torch.zeros_like(top), top)
    x.sub_(top).exp_()
    total = x.sum(-1, keepdim=True)
    out = torch.matmul(x.reshape(S, Hkv, G * Mq, Mk), v).reshape(S, Hkv, G, Mq, D) / torch.where(total > 0, total, torch.ones_like(total))
    lse = (top + total.log())[..., 0]
    return out.permute(0, 3, 1, 2, 4).reshape(S, Mq, Hq, D), lse.permute(0, 3, 1, 2).reshape(S, Mq, Hq)


def _plain_attention(st):
    case, q = st["case"], st["q"]
    cu, kv_len, T, S = st["cu_q"], st["kv_len"], q.shape[0], len(st["kv_len"])
    q_len = cu[1:] - cu[:-1]
    if case["kind"] == "paged":
        table = st["table"][:, :-(-max(st["max_kv"], 1) // case["page"])].long()
        k, v = (p[table].permute(0, 2, 1, 3, 4).float().reshape(S, case["Hkv"], -1, D)[:, :, :st["max_kv"]] for p in (st["k_pages"], st["v_pages"]))
    else:
        at = (cu[:-1, None] + torch.arange(st["max_kv"], device="cuda")).clamp_(max=T - 1).long()
        k, v = (x[at].transpose(1, 2).float().contiguous() for x in (st["k"], st["v"]))
    at = (cu[:-1, None] + torch.arange(st["max_q"], device="cuda")).clamp_(max=T - 1).long()
    out, lse = _softmax_attention(q[at], k, v, q_len, kv_len, case)
    seq, i = _sequence_of(cu, T)
    return out[seq, i.long()].to(q.dtype), lse[seq, i.long()].contiguous()


def run(st):
    if own:
        return _run_own(st)
    return _plain_rope(st) if st["case"]["kind"] == "rope" else _plain_attention(st)


def _seen_by(case, q, kv):
    """(pairs of a row and a token it sees, tokens that any row sees) of one sequence."""
    if not case["causal"]:
        return q * kv, kv if q else 0
    pairs = 0
    for p in range(kv - q, kv):
        n = p + 1
        pairs += min(n, case["window"] + min(case["sink"], max(0, n - case["window"]))) if case["window"] else n
    first = kv - q + 1 - case["window"] if case["window"] else 0
    return pairs, kv - max(0, first) + min(case["sink"], max(0, first)) if q else 0


def work(case):
    q, kv = _lens(case)
    es, T, Hq, Hkv = 2 if case["dtype"] == "bf16" else 4, sum(q), case["Hq"], case["Hkv"]
    if case["kind"] == "rope":
        return {"bytes": 2 * T * (Hq + 2 * Hkv) * D * es, "flops": 3 * T * (Hq + Hkv) * case["rotary"]}
    seen = [_seen_by(case, a, b) for a, b in zip(q, kv)]
    return {"bytes": (2 * T * Hq + 2 * Hkv * sum(n for _, n in seen)) * D * es + 4 * T * Hq, "flops": 4 * D * Hq * sum(p for p, _ in seen)}


def exact(case, seed):
    st = _inputs(case, seed)
    q, kv = _lens(case)
    if case["kind"] == "rope":
        return _exact_rope(case, st, q, kv)
    Hkv, G = case["Hkv"], case["Hq"] // case["Hkv"]
    out = torch.zeros(sum(q), case["Hq"], D, dtype=torch.float64, device="cuda")
    lse = torch.full((sum(q), case["Hq"]), -math.inf, dtype=torch.float64, device="cuda")
    row = tok = 0
    for s, (a, n) in enumerate(zip(q, kv)):
        if a and n:
            place = torch.arange(n - a, n, device="cuda")[:, None]
            t = torch.arange(n, device="cuda")[None]
            hidden = t > place if case["causal"] else torch.zeros(a, n, dtype=torch.bool, device="cuda")
            if case["window"]:
                hidden |= (t <= place - case["window"]) & (t >= case["sink"])
            for h in range(Hkv):
                if case["kind"] == "paged":
                    pages = st["table"][s, :-(-n // case["page"])].long()
                    kh, vh = (p[pages, h].reshape(-1, D)[:n].double() for p in (st["k_pages"], st["v_pages"]))
                else:
                    kh, vh = (x[tok:tok + n, h].double() for x in (st["k"], st["v"]))
                for j in range(h * G, (h + 1) * G):
                    logits = st["q"][row:row + a, j].double() @ kh.T.contiguous() / math.sqrt(D)
                    logits.masked_fill_(hidden, -math.inf)
                    lse[row:row + a, j] = torch.logsumexp(logits, 1)
                    ok = lse[row:row + a, j] > -math.inf
                    weights = logits.sub_(torch.where(ok, lse[row:row + a, j], 0.0)[:, None]).exp_()
                    out[row:row + a, j] = weights @ vh
        row += a
        tok += n
    return out, lse


def _exact_rope(case, st, q, kv):
    half, r = case["pairing"] == "half", case["rotary"]
    freq = torch.tensor(_frequencies(r, case["scaling"])[0], dtype=torch.float64, device="cuda")
    wheel = torch.polar(torch.full_like(freq, st["magnitude"])[None].expand(sum(q), -1).contiguous(), st["positions"].double()[:, None] * freq)[:, None]
    def turned(x):
        x = x.double()
        z = torch.complex(x[..., :r // 2].contiguous(), x[..., r // 2:r].contiguous()) if half else torch.complex(x[..., 0:r:2].contiguous(), x[..., 1:r:2].contiguous())
        z = z * wheel
        x[..., :r] = torch.cat((z.real, z.imag), -1) if half else torch.view_as_real(z).flatten(-2)
        return x
    k_pages, v_pages, k = st["k_pages"].double(), st["v_pages"].double(), turned(st["k"])
    row = 0
    for s, (a, n) in enumerate(zip(q, kv)):
        at = torch.arange(n - a, n, device="cuda")
        page = st["table"][s][at // case["page"]].long()
        k_pages[page, :, at % case["page"]] = k[row:row + a]
        v_pages[page, :, at % case["page"]] = st["v"][row:row + a].double()
        row += a
    return turned(st["q"]), k_pages, v_pages
