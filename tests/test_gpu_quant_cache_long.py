"""GPU parity of quantised caches, head norms and reading back where calls are large or uneven: batches with one long context, chunks of a few thousand tokens, many heads, long reads."""
import numpy as np
import pytest
import torch

import paper_2508_17892_amd as il
from oracle import quant_cache as oq
from test_gpu_attention import DT, Paged, _announce, _f64
from test_gpu_quant_cache import AXES3, BASE, Quant, _near, _states, _turned, _weights

pytestmark = pytest.mark.gpu


def uneven(long_at):
    """Lengths of 130 contexts."""
    return [9000 if i == long_at else 1 + 7 * i % 50 for i in range(130)]


@pytest.mark.parametrize("dtype,layout,long_at", [("bf16", "head", 0), ("bf16", "token", 129), ("f32", "head", 64)])
@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
def test_one_long_context_among_many_short_ones(fmt, dtype, layout, long_at):
    """More lists than two for each compute unit, and one of them far longer than its share of the work."""
    _announce(f"quantised, one long context among 130 {fmt} {dtype} {layout}")
    x = Quant(fmt, [1] * 130, uneven(long_at), 8, 8, 64, dtype, layout, seed=long_at)
    out, lse = x.attend()
    torch.cuda.synchronize()
    x.check(out, lse)
    again, lse2 = x.attend()
    assert torch.equal(out, again) and torch.equal(lse, lse2)
    x.check(*x.attend(workspace=torch.empty(0, dtype=torch.uint8, device="cuda")))


# ------------------------------------------------------------------------------------------------ filling a cache: every kernel, several steps of query heads

# q_lens, kv_lens, Hq, Hkv, rows of no sequence (in front, behind)
FILL_SHAPES = {
    "few": ([1, 2, 0, 1], [1, 900, 5, 64], 64, 8, (0, 0)),             # eight wavefronts a token, one goes from queries to keys
    "512": ([300, 212], [500, 300], 12, 3, (0, 0)),
    "513": ([513], [513], 28, 4, (0, 0)),                              # four wavefronts
    "chunks": ([600, 0, 423], [700, 3, 423], 28, 4, (2, 3)),
    "chunk": ([1028], [1500], 32, 8, (0, 0)),
    "wide": ([1028], [1028], 64, 8, (0, 1)),
    "4095": ([4000, 95], [4000, 100], 9, 1, (0, 0)),
    "4096": ([4096], [4100], 9, 1, (0, 0)),                            # one
    "many": ([2500, 1700], [2500, 1800], 28, 4, (1, 2)),
    "many, 64/8": ([4100], [4100], 64, 8, (0, 0)),
}
PAIRINGS = (("half", 128), ("half", 64), ("interleaved", 96))
FILL_CALLS = [(shape, dtype, fmt, *PAIRINGS[i]) for dtype in ("bf16", "f32") for fmt in ("plain", "fp8", "fp4") for i in range(3) for shape in ("few", "chunks", "many")]
FILL_CALLS += [(shape, "bf16", fmt, *PAIRINGS[i]) for i, fmt in enumerate(("fp8", "fp4", "plain")) for shape in ("512", "513", "chunk", "wide", "4095", "4096")]
FILL_CALLS += [("many, 64/8", "bf16", "fp8", "half", 128), ("wide", "f32", "fp4", "half", 128)]


def _blank(fmt, kv_lens, Hq, Hkv, page, dtype, layout):
    """A quantised cache of such lengths with nothing in it: the tables alone are made, and pages of ones."""
    x = Paged([0] * len(kv_lens), [0] * len(kv_lens), Hq, Hkv, page, dtype, layout)
    need = [-(-n // page) for n in kv_lens]
    total = sum(need) + 2
    order = torch.randperm(total, generator=torch.Generator().manual_seed(total)).int()
    x.table = torch.full((len(kv_lens), max(need)), -7, dtype=torch.int32)
    for s, m in enumerate(need):
        x.table[s, :m] = order[sum(need[:s]):sum(need[:s]) + m]
    x.dev.update(table=x.table.cuda(), kv_len=torch.tensor(kv_lens, dtype=torch.int32).cuda())

    def pages(width):
        t = torch.ones((total, page, Hkv, width) if layout == "token" else (total, Hkv, page, width), dtype=torch.uint8, device="cuda")
        return t.permute(0, 2, 1, 3) if layout == "token" else t

    x.kp, x.vp, x.ks, x.vs = (pages(w) for w in ((128,) * 2 if fmt == "fp8" else (64,) * 2) + (4, 4))
    if fmt == "fp8":
        x.kp, x.vp = x.kp.view(torch.float8_e4m3fn), x.vp.view(torch.float8_e4m3fn)
    x.cache = lambda: il.QuantKV(x.kp, x.vp, x.ks, x.vs, x.dev["table"], x.dev["kv_len"], x.dev["cu"])
    return x


@pytest.mark.parametrize("shape,dtype,fmt,pairing,rotary", FILL_CALLS)
def test_fill_of_every_size(shape, dtype, fmt, pairing, rotary):
    _announce(f"fill, {shape} {dtype} {fmt} {pairing} {rotary}")
    q_lens, kv_lens, Hq, Hkv, (front, behind) = FILL_SHAPES[shape]
    n, page, axes = sum(q_lens), 16, 3 if fmt != "fp4" else 1
    T = front + n + behind
    args = (kv_lens, Hq, Hkv, page, dtype, "token" if pairing == "half" else "head")
    x = Paged([0] * len(kv_lens), *args, fill=0.5) if fmt == "plain" else _blank(fmt, *args)
    x.dev["cu"] = torch.tensor([front] + list(front + np.cumsum(q_lens)), dtype=torch.int32).cuda()
    fused = _states(T, Hq, Hkv, dtype, T + rotary)
    q, k, v = fused[:, :Hq], fused[:, Hq:Hq + Hkv], fused[:, Hq + Hkv:]
    qw, kw = _weights(dtype, rotary, 0)
    f = il.ilre_rope_frequencies(rotary, BASE)
    places = np.concatenate([np.full(front, 3)] + [np.arange(m - a, m) for a, m in zip(q_lens, kv_lens)] + [np.full(behind, 5)])
    pos = places[None] if axes == 1 else np.stack((places, places // 7 - 20, places % 31 + 5))
    table = (0,) * (rotary // 2) if axes == 1 else AXES3[rotary // 2]
    dev, got = fused.cuda(), torch.full((T, Hq, 128), 9.0, dtype=DT[dtype], device="cuda")
    before = {name: getattr(x, name).clone() for name in ("kp", "vp") + (("ks", "vs") if fmt != "plain" else ())}
    il.ilre_norm_rope_append(dev[:, :Hq], dev[:, Hq:Hq + Hkv], dev[:, Hq + Hkv:], x.cache(), f, None if axes == 1 else torch.from_numpy(pos).int().cuda(),
                             norms=il.HeadNorms(qw.cuda(), kw.cuda(), eps=1e-6), axes=None if axes == 1 else table, q_out=got,
                             pairing=il.ILRE_ROPE_HALF if pairing == "half" else il.ILRE_ROPE_INTERLEAVED)
    torch.cuda.synchronize()
    mine = slice(front, front + n)
    assert (got[:front] == 9).all() and (got[front + n:] == 9).all()
    pos = pos[:, mine]
    sizes = [np.abs(oq.norm(_f64(t[mine]), _f64(w), 1e-6)).max(-1, keepdims=True) * 2 for t, w in ((q, qw), (k, kw))]
    _near(got[mine], _turned(q[mine], qw, pos, table, f, pairing, 0), sizes[0], dtype)
    want_k, want_v = _turned(k[mine], kw, pos, table, f, pairing, 0), _f64(v[mine])
    seq, places = np.repeat(np.arange(len(q_lens)), q_lens), places[mine]
    page_at, cell = x.table[seq, places // page].long().cuda(), torch.from_numpy(places % page).cuda()
    if fmt == "plain":
        _near(x.kp[page_at, :, cell], want_k, sizes[1], dtype)
        assert torch.equal(x.vp[page_at, :, cell].cpu(), v[mine])
    else:
        for pages, scales, want in ((x.kp, x.ks, want_k), (x.vp, x.vs, want_v)):
            codes, sc = oq.store(want, fmt)
            assert np.array_equal(scales[page_at, :, cell].cpu().numpy(), sc)
            stored = pages.view(torch.uint8)[page_at, :, cell].cpu().numpy()
            assert np.array_equal(stored, codes), (int((stored != codes).sum()), codes.size)
    for name, old in before.items():  # nothing else was touched
        a, b = (t.view(torch.uint8) if t.dtype == torch.float8_e4m3fn else t for t in (old, getattr(x, name)))
        a[page_at, :, cell] = b[page_at, :, cell]
        assert torch.equal(a, b), name


TURNS = [(1, 64), (512, 9), (600, 28), (4095, 3), (4200, 28)]


@pytest.mark.parametrize("T,H", TURNS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_norm_rope_of_every_size(T, H, dtype):
    _announce(f"norm_rope {T} {H} {dtype}")
    x = _states(T, H, 1, dtype, T)[:, :H]
    w = _weights(dtype, T, 1)[0]
    pos = np.stack((np.arange(T) + 1000, np.arange(T) // 24, np.arange(T) % 24 - 7))
    for pairing, rotary in PAIRINGS:
        f, axes = il.ilre_rope_frequencies(rotary, BASE), AXES3[rotary // 2]
        size = np.abs(oq.norm(_f64(x), _f64(w), 1e-6, 1.0)).max(-1, keepdims=True) * 2
        kw = dict(norms=il.HeadNorms(w.cuda(), eps=1e-6, offset=1.0), axes=axes, pairing=il.ILRE_ROPE_HALF if pairing == "half" else il.ILRE_ROPE_INTERLEAVED)
        got = il.ilre_norm_rope(x.cuda(), f, torch.from_numpy(pos).int().cuda(), **kw)
        _near(got, _turned(x, w, pos, axes, f, pairing, 1.0), size, dtype)
        y = x.cuda()
        il.ilre_norm_rope(y, f, torch.from_numpy(pos).int().cuda(), out=y, **kw)
        assert torch.equal(y, got)


# ------------------------------------------------------------------------------------------------ reading back: several rows a lane

READ_ROWS = {
    "few long": ([700, 0, 64, 1, 300, 0], [20000, 0, 9000, 3, 3990, 0], 8),
    "many short": ([i % 9 for i in range(1500)], [(7 * i) % 46 for i in range(1500)], 8),
    "one head": ([900, 33], [200000, 62300], 1),
}
READS = [("few long", fmt, dtype) for fmt in ("plain", "fp8", "fp4") for dtype in ("bf16", "f32")] + [("many short", "fp8", "bf16"), ("one head", "fp4", "bf16")]


@pytest.mark.parametrize("rows,fmt,dtype", READS)
def test_long_reads(rows, fmt, dtype):
    _announce(f"long read, {rows} {fmt} {dtype}")
    lens, rows, H = READ_ROWS[rows]
    S, page = len(lens), 16
    args = ([0] * S, lens, H, H, page, dtype, "head" if fmt == "fp8" else "token")
    x = Paged(*args, seed=3) if fmt == "plain" else Quant(fmt, *args, seed=3)
    x.dev["table"][0, 0] = -1  # the first sequence's first tokens are on no page
    out_type = DT[dtype]
    k, v = ([t.to(out_type) for t in s] for s in (x.k, x.v))
    for t in (k, v):
        t[0][:page] = 0
    # every sequence's tokens, and behind them a row of zeros for those that are not there
    begin = np.concatenate(([0], np.cumsum(np.array(lens) + 1)))[:-1]
    k, v = (torch.cat([torch.cat((t[s], torch.zeros(1, H, 128, dtype=out_type))) for s in range(S)]) for t in (k, v))
    T, front, behind = sum(rows), 2, 3
    seq = np.repeat(np.arange(S), rows)
    rng = np.random.default_rng(0)
    lengths = np.array(lens)[seq]
    last = lengths - np.array(rows)[seq] + np.arange(T) - np.concatenate(([0], np.cumsum(rows)))[seq]
    for tokens in (rng.integers(-3, lengths + 5), None):
        at = last if tokens is None else tokens
        where = torch.from_numpy(begin[seq] + np.where((at >= 0) & (at < lengths), at, lengths))
        x.dev["cu"] = torch.tensor([front] + list(front + np.cumsum(rows)), dtype=torch.int32).cuda()
        given = None if tokens is None else torch.from_numpy(np.concatenate((np.zeros(front), tokens, np.zeros(behind)))).int().cuda()
        for layout in ("token", "head"):
            out = [torch.full((T + front + behind, H, 128) if layout == "token" else (H, T + front + behind, 128), 9.0, dtype=out_type, device="cuda") for _ in range(2)]
            view = out if layout == "token" else [t.transpose(0, 1) for t in out]
            il.ilre_cache_read(x.cache(), T + front + behind, given, k_out=view[0], v_out=view[1])
            torch.cuda.synchronize()
            for got, states in zip(view, (k, v)):
                assert torch.equal(got[front:front + T].cpu(), states[where]) and (got[:front] == 9).all() and (got[front + T:] == 9).all()


# ------------------------------------------------------------------------------------------------ far positions

FAR = (999983, 1000003, 65000011, 2 ** 30 + 7, 2 ** 31 - 1, -(2 ** 31))


def next_to_a_border(position, inv_freq, rng, n=1 << 16):
    """fp32 (x1, x2) whose first channel, turned to the position, lies so near to 17, halfway between two codes, that an angle rounded to fp64 on the way (as turns, product and rest each rounded) puts
    it on the other side; None where the search finds none."""
    (cos, sin), turns = oq.angle(position, inv_freq), inv_freq / (2 * np.pi)
    part = position * turns - np.rint(position * turns)
    off_cos, off_sin = np.cos(2 * np.pi * part), np.sin(2 * np.pi * part)
    if abs(cos) < 0.3:
        return None
    x2 = rng.uniform(16, 32, n).astype(np.float32).astype(np.float64)
    x1 = ((17 + x2 * sin) / cos).astype(np.float32).astype(np.float64)
    real, other = x1 * cos - x2 * sin - 17, x1 * off_cos - x2 * off_sin - 17
    # (fp64 itself: a few times 2^-53 of products of up to 170)
    hits = np.flatnonzero((real * other < 0) & (np.minimum(np.abs(real), np.abs(other)) > 2.0 ** -42))
    return (x1[hits[0]], x2[hits[0]]) if len(hits) else None


def far_states(pairing, rotary, inv_freq, seed):
    """Keys [positions, 1, 128] of which channels lie next to borders of codes under a scale of one, and how many do."""
    rng = np.random.default_rng(seed)
    x, found = np.zeros((len(FAR), 1, 128)), 0
    for t, p in enumerate(FAR):
        for j in range(min(rotary // 2, 30)):
            got = next_to_a_border(p, inv_freq[j], rng)
            a, b = (j, j + rotary // 2) if pairing == "half" else (2 * j, 2 * j + 1)
            if got and (pairing == "half" or j < 16):
                x[t, 0, a], x[t, 0, b] = got
                found += 1
        # the block's largest magnitude: not turned, or turned from where it comes out as the first of its pair
        if rotary < 128:
            x[t, 0, 20 + rotary // 4] = 300
        else:
            cos, sin = oq.angle(p, inv_freq[31])
            x[t, 0, 31], x[t, 0, 31 + 64] = np.float32(300 * cos), np.float32(-300 * sin)
    return torch.from_numpy(x).float(), found


@pytest.mark.parametrize("pairing,rotary", [("half", 128), ("half", 16), ("interleaved", 16)])
def test_keys_at_far_positions_fall_on_their_side_of_a_border(pairing, rotary):
    """What a cache holds is a function of the states alone, at a million tokens and at the last position there is."""
    _announce(f"fill, far positions {pairing} {rotary}")
    f = il.ilre_rope_frequencies(rotary, 500000.0)
    inv_freq = np.array(f.inv_freq)[:rotary // 2]
    k, found = far_states(pairing, rotary, inv_freq, rotary)
    assert found >= 6
    n = len(FAR)
    for repeat in (1, 700 // n, 4100 // n + 1):  # each kind of kernel
        T = n * repeat
        x = _blank("fp8", [T], 4, 1, 16, "f32", "head")
        x.dev["cu"] = torch.tensor([0, T], dtype=torch.int32).cuda()
        states, pos = k.repeat(repeat, 1, 1).cuda(), torch.tensor(FAR * repeat, dtype=torch.int64).int().cuda()
        il.ilre_norm_rope_append(None, states, None, x.cache(), f, pos, pairing=il.ILRE_ROPE_HALF if pairing == "half" else il.ILRE_ROPE_INTERLEAVED)
        want = oq.rope_axes(_f64(k), np.array(FAR)[None], [0] * (rotary // 2), inv_freq, 1.0, pairing)
        codes, scales = oq.store(want, "fp8")
        assert (scales[:, 0, 0] == 127).all()
        t = np.arange(T)
        at, cell = x.table[0, t // 16].long().cuda(), torch.from_numpy(t % 16).cuda()
        got = x.kp.view(torch.uint8)[at, :, cell].cpu().numpy()
        bad = got != np.tile(codes, (repeat, 1, 1))
        assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:5].tolist())
        assert np.array_equal(x.ks[at, :, cell].cpu().numpy(), np.tile(scales, (repeat, 1, 1)))


@pytest.mark.parametrize("n,kv,Hq,Hkv,dtype", [(1, 300, 8, 2, "bf16"), (1, 9000, 8, 2, "f32"), (7, 300, 8, 2, "bf16"), (200, 600, 8, 2, "bf16"), (200, 600, 8, 2, "f32"), (200, 600, 64, 8, "bf16")])
@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
def test_blocks_that_stand_for_nan(fmt, n, kv, Hq, Hkv, dtype):
    """A block marked by the fill (byte 255, codes of zero) that rows see: nothing finite comes of it."""
    _announce(f"byte 255 that is seen, {fmt} {n} of {kv} {Hq}/{Hkv} {dtype}")
    G, t = Hq // Hkv, kv // 3  # a token that all rows see
    for name in ("k", "v"):
        x = Quant(fmt, [n], [kv], Hq, Hkv, 16, dtype, seed=1)
        at = (int(x.table[0, t // 16]), 1, t % 16)
        codes, scales = x.host[name]
        codes[at][slice(32, 64) if fmt == "fp8" else slice(16, 32)] = 0
        scales[at][1] = 255
        x.upload()
        out, lse = x.attend()
        torch.cuda.synchronize()
        want, want_lse = torch.zeros(n, Hq, 128, dtype=torch.bool), torch.zeros(n, Hq, dtype=torch.bool)
        want[:, G:2 * G, slice(None) if name == "k" else slice(32, 64)] = True
        want_lse[:, G:2 * G] = name == "k"
        assert torch.equal(torch.isnan(out).cpu(), want) and torch.equal(torch.isnan(lse).cpu(), want_lse)
        assert torch.isfinite(out[~want.cuda()]).all() and torch.isfinite(lse[~want_lse.cuda()]).all()


@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
@pytest.mark.parametrize("q_len", [1, 9])
def test_queries_up_to_the_largest_float(fmt, q_len):
    """fp32 queries beyond what bf16, of which three parts make one, rounds to a number; their logits are small."""
    _announce(f"largest queries {fmt} {q_len}")
    x = Quant(fmt, [q_len], [200], 8, 2, 16, "f32", seed=3)
    codes, scales = oq.store(_f64(x.k[0]) * 2.0 ** -10, fmt)  # (products that fp32 holds)
    t = torch.arange(200)
    for part, new in zip(x.host["k"], (codes, scales)):
        part[x.table[0, t // 16].long(), :, t % 16] = torch.from_numpy(new)
    x.k[0] = torch.from_numpy(oq.read(codes, scales, fmt))
    x.upload()
    top = torch.finfo(torch.float32).max
    x.q[:, :, 5], x.q[:, ::2, 70] = top, -top
    x.q[:, 1, 5] = top * (1 - 2.0 ** -8)
    x.dev["q"] = x.q.cuda()
    out, lse = x.attend(scale=2.0 ** -118)
    torch.cuda.synchronize()
    x.check(out, lse, scale=2.0 ** -118)


@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
@pytest.mark.parametrize("power", [-140, -132, -126, -118])
def test_keys_around_the_least_scale(fmt, power):
    """Keys below 2^-126 are rounded to multiples of 2^-149 on their way to a code: what lies further than that from a border falls on its side of it."""
    _announce(f"fill, keys of 2^{power} {fmt}")
    T = 64
    k = (torch.randn(T, 2, 128, generator=torch.Generator().manual_seed(-power), dtype=torch.double) * 2.0 ** power).float()
    x = _blank(fmt, [T], 4, 2, 16, "f32", "head")
    x.dev["cu"] = torch.tensor([0, T], dtype=torch.int32).cuda()
    f = il.ilre_rope_frequencies(128, BASE)
    il.ilre_norm_rope_append(None, k.cuda(), k.cuda(), x.cache(), f)
    want = oq.rope_axes(_f64(k), np.arange(T)[None], [0] * 64, np.array(f.inv_freq)[:64])
    t = np.arange(T)
    at, cell = x.table[0, t // 16].long().cuda(), torch.from_numpy(t % 16).cuda()
    for pages, scales, y, off in ((x.kp, x.ks, want, 2.0 ** -149), (x.vp, x.vs, _f64(k), 0.0)):
        got, sc = pages.view(torch.uint8)[at, :, cell].cpu().numpy(), scales[at, :, cell].cpu().numpy()
        value = oq.read(got, sc, fmt)
        assert np.array_equal(sc, oq.store(y, fmt)[1])
        low, high = (oq.read(*oq.store(np.where(np.abs(y) > 2 * off, np.sign(y) * (np.abs(y) + d), y), fmt), fmt) for d in (-off, off))
        sure = low == high
        assert np.array_equal(value[sure], low[sure]) and sure.mean() > 0.99
