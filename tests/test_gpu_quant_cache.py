"""GPU parity of head norms, axes, quantised caches and drafted trees, through the C ABI, against the fp64 oracle on the same inputs.

A quantised cache's bytes are a function of the states (rounded once, from fp64): they have to be the oracle's.  Attention over it is held to the tolerances of attention over a
cache of the states' type, on the numbers that the codes stand for: these are exact in bf16 and fp32, so that the same products are rounded in the same places.
"""
import numpy as np
import pytest
import torch

import paper_2508_17892_amd as il
from oracle import attention as oa
from oracle import quant_cache as oq
from test_gpu_attention import CASES, DT, HALF, Paged, _announce, _check, _f64, _rope_check

pytestmark = pytest.mark.gpu

BASE = 10000.0
AXES3 = {n: tuple(0 if j < n // 4 else 1 + j % 2 for j in range(n)) for n in (8, 32, 48, 64)}


def _i32(*x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _u8(t):
    return t.view(torch.uint8).cpu().numpy()


class Quant(Paged):
    """Random sequences in a quantised cache; everything that is nobody's token holds NaN codes and scales."""

    def __init__(self, fmt, *args, **kw):
        super().__init__(*args, **kw)
        self.fmt = fmt
        self.layout = "head" if self.kp.is_contiguous() else "token"
        n, Hkv, P, _ = self.kp.shape
        blank = lambda width: torch.full((n, P, Hkv, width) if self.layout == "token" else (n, Hkv, P, width), 255, dtype=torch.uint8)  # noqa: E731
        self.host = {}
        for name in ("k", "v"):
            pages, scales = blank(128 if fmt == "fp8" else 64), blank(4)
            view = [t.permute(0, 2, 1, 3) if self.layout == "token" else t for t in (pages, scales)]
            states = getattr(self, name)
            for s, x in enumerate(states):
                codes, sc = oq.store(_f64(x), fmt)
                t = torch.arange(len(x))
                at = (self.table[s, t // P].long(), slice(None), t % P)
                view[0][at], view[1][at] = torch.from_numpy(codes), torch.from_numpy(sc)
                states[s] = torch.from_numpy(oq.read(codes, sc, fmt))
            self.host[name] = pages, scales
        self.upload()

    def upload(self):
        for name in ("k", "v"):
            pages, scales = (t.cuda() for t in self.host[name])
            if self.fmt == "fp8":
                pages = pages.view(torch.float8_e4m3fn)
            if self.layout == "token":
                pages, scales = pages.permute(0, 2, 1, 3), scales.permute(0, 2, 1, 3)
            setattr(self, name + "p", pages)
            setattr(self, name + "s", scales)

    def cache(self):
        return il.QuantKV(self.kp, self.vp, self.ks, self.vs, self.dev["table"], self.dev["kv_len"], self.dev["cu"])


# ------------------------------------------------------------------------------------------------ attention over a quantised cache

ATTENTION = CASES + [
    ([300], [900], 64, 8, 16, "head", "bf16", {}),                             # 256 rows a workgroup
    ([1024, 700], [3000, 700], 32, 8, 64, "head", "bf16", {}),
    ([600], [600], 64, 8, 32, "token", "bf16", dict(sink=4, window=200)),
    ([1], [70001], 8, 1, 64, "head", "bf16", {}),
    ([7, 5], [3000, 900], 8, 2, 16, "head", "bf16", {}),                       # 32 rows
    ([7], [3000], 8, 2, 64, "token", "bf16", dict(sink=4, window=700)),
    ([2100], [2100], 32, 8, 64, "head", "bf16", dict(sink=4, window=128)),     # 256 rows, whole
    ([2, 3], [60, 40], 8, 2, 16, "head", "f32", {}),
    ([3], [900], 8, 2, 32, "head", "f32", dict(sink=4, window=100)),
    ([40], [40], 8, 2, 16, "head", "f32", {}),
]


@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
@pytest.mark.parametrize("q_lens,kv_lens,Hq,Hkv,page,layout,dtype,mask", ATTENTION)
def test_attention(fmt, q_lens, kv_lens, Hq, Hkv, page, layout, dtype, mask):
    _announce(f"quantised {fmt} {q_lens} of {kv_lens} {Hq}/{Hkv} page {page} {layout} {dtype} {mask}")
    x = Quant(fmt, q_lens, kv_lens, Hq, Hkv, page, dtype, layout, seed=sum(kv_lens) + Hq)
    out, lse = x.attend(**mask)
    torch.cuda.synchronize()
    x.check(out, lse, **mask)
    again, lse2 = x.attend(**mask)
    assert torch.equal(out, again) and torch.equal(lse, lse2)
    for ws in (torch.empty(0, dtype=torch.uint8, device="cuda"), torch.empty(sum(q_lens) * Hq * 516 * 2 + 256, dtype=torch.uint8, device="cuda")):
        x.check(*x.attend(workspace=ws, **mask), **mask)


# Heads side by side, and so much work (as promised; it goes into how a call is cut up, not into what comes out) that a workgroup takes several.
BESIDE = [
    # format (1: 8 bits), q_lens, kv_lens, Hq, Hkv, page, mask, longest and total promised, heads a workgroup
    (1, [1], [5000], 8, 8, 64, {}, 70000, 70000, 2),
    (1, [2, 1, 0, 4], [700, 1031, 9, 64], 16, 4, 16, {}, 300000, 300000, 2),
    (1, [1, 3] * 64, [500, 100, 45, 3] * 32, 16, 8, 32, dict(sink=4, window=300), 700, 128 * 700, 2),
    (1, [1] * 70, [300, 17, 1, 0, 95, 512, 33] * 10, 12, 6, 16, {}, 512, 400000, 2),           # whole
    (1, [1], [9000], 32, 8, 64, {}, 1000000, 1000000, 4),
    (1, [2, 1, 0, 4], [700, 1031, 9, 64], 16, 4, 16, {}, 1000000, 4000000, 4),
    (1, [1] * 150, [300, 17, 1] * 50, 16, 8, 16, {}, 300, 300 * 1000, 4),
    (2, [1], [9000], 32, 8, 64, {}, 1000000, 1000000, 4),
    (2, [3, 1, 0, 4], [700, 1031, 9, 64], 12, 4, 16, {}, 1000000, 4000000, 4),
    (2, [1] * 150, [300, 17, 1] * 50, 16, 8, 16, {}, 300, 300 * 1000, 4),
]


@pytest.mark.parametrize("fmt,q_lens,kv_lens,Hq,Hkv,page,mask,most,total,heads", BESIDE)
def test_several_heads_a_workgroup(fmt, q_lens, kv_lens, Hq, Hkv, page, mask, most, total, heads):
    _announce(f"quantised, {heads} heads a workgroup, format {fmt} {len(q_lens)} sequences {Hq}/{Hkv} page {page} {mask}")
    x = Quant({1: "fp8", 2: "fp4"}[fmt], q_lens, kv_lens, Hq, Hkv, page, "bf16", "token", seed=sum(kv_lens))
    run = lambda **kw: il.ilre_paged_attention(x.dev["q"], x.cache(), max_q=max(q_lens), max_kv=most, total_kv=total, **mask, **kw)  # noqa: E731
    out, lse = run()
    torch.cuda.synchronize()
    x.check(out, lse, **mask)
    again, lse2 = run()
    assert torch.equal(out, again) and torch.equal(lse, lse2)
    x.check(*run(workspace=torch.empty(0, dtype=torch.uint8, device="cuda")), **mask)
    if len(q_lens) == 1:
        absent = [np.zeros(kv_lens[0], bool)]
        for col in (0, 3, kv_lens[0] // page):
            x.dev["table"][0, col] = -1
            absent[0][col * page:col * page + page] = True
        x.check(*run(), absent=absent, **mask)


@pytest.mark.parametrize("q_len,mask", [(1, {}), (50, {}), (200, {}), (200, dict(sink=4, window=64)), (1, dict(sink=20, window=64))])
@pytest.mark.parametrize("fmt,dtype", [("fp8", "bf16"), ("fp4", "bf16"), ("fp8", "f32")])
def test_entries_that_name_no_page(q_len, mask, fmt, dtype):
    _announce(f"quantised, absent pages, {fmt} {dtype} {q_len} new {mask}")
    x = Quant(fmt, [q_len, 3], [1000, 60], 8, 2, 16, dtype, seed=q_len)
    absent = [np.zeros(1000, bool), np.zeros(60, bool)]
    for col, entry in {0: -1, 7: 1 << 30, 20: x.kp.shape[0], 33: -2 ** 31, 61: -5}.items():
        x.dev["table"][0, col] = entry
        absent[0][col * 16:col * 16 + 16] = True
    x.check(*x.attend(**mask), absent=absent, **mask)
    x.dev["table"][0] = -1
    absent[0][:] = True
    x.check(*x.attend(**mask), absent=absent, **mask)


@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
def test_freed_pages_hold_anything(fmt):
    """Between the sink part and the window nothing is looked at: NaN codes and scales there, or no pages."""
    _announce(f"quantised, freed pages {fmt}")
    for q_len in (1, 30, 300):
        x = Quant(fmt, [q_len], [2000], 8, 2, 16, "bf16", seed=5)
        first = 2000 - q_len - 100 + 1
        for t in range(4, first):
            for name in ("k", "v"):
                for part in x.host[name]:
                    part[x.table[0, t // 16], :, t % 16] = 255
        x.upload()
        freed = [c for c in range(125) if c * 16 >= 16 and c * 16 + 16 <= first]
        out, lse = x.attend(sink=4, window=100)
        x.check(out, lse, sink=4, window=100)
        x.dev["table"][0, freed] = -1
        out2, lse2 = x.attend(sink=4, window=100)
        assert torch.equal(out, out2) and torch.equal(lse, lse2)


@pytest.mark.parametrize("q_len,kv", [(1, 3000), (64, 3000), (300, 3000)])
@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
def test_late_tokens_that_outweigh_everything_before(q_len, kv, fmt):
    _announce(f"quantised, rising logits, {q_len} of {kv} {fmt}")
    for sign in (1, -1):
        x = Quant(fmt, [q_len], [kv], 8, 2, 16, "bf16", seed=7)
        step = (torch.linspace(-1, 1, kv)[:, None, None] * sign * 40).expand(kv, 2, 128).double().numpy()
        codes, scales = oq.store(step, fmt)
        t = torch.arange(kv)
        for part, new in zip(x.host["k"], (codes, scales)):
            part[x.table[0, t // 16].long(), :, t % 16] = torch.from_numpy(new)
        x.k[0] = torch.from_numpy(oq.read(codes, scales, fmt))
        x.upload()
        x.q = (x.q.float() * 0.1 + 1).bfloat16()
        x.dev["q"] = x.q.cuda()
        x.check(*x.attend())


def test_lengths_promised_otherwise_and_beyond_the_table():
    _announce("quantised, lengths")
    x = Quant("fp8", [40, 1, 90], [900, 333, 90], 8, 2, 16, "bf16", seed=3)
    for max_q, max_kv, total in ((1, 1, 1), (1, 16, 5000), (90, 100000, 0), (4000, 900, 100)):
        x.check(*il.ilre_paged_attention(x.dev["q"], x.cache(), max_q=max_q, max_kv=max_kv, total_kv=total))
    x = Quant("fp4", [3], [64], 8, 2, 16, "bf16", seed=6)
    x.dev["kv_len"].fill_(1 << 30)
    x.check(*x.attend())
    x.dev["kv_len"].fill_(-5)
    out, lse = x.attend()
    assert (out == 0).all() and (lse == -float("inf")).all()


def test_boundaries_that_do_not_ascend_stay_within_the_tensors():
    _announce("quantised, unordered boundaries")
    x = Quant("fp8", [40] * 3, [300, 41, 1000], 8, 2, 16, "bf16", seed=21)
    guard = torch.full((140, 8, 128), 9.0, device="cuda").bfloat16()
    kv = torch.full((140, 2, 128), 9.0, device="cuda").bfloat16()
    tree = torch.full((120, 4), -1, dtype=torch.int32, device="cuda")
    f = il.ilre_rope_frequencies(128, 1e4)
    for cu in ([0, 90, 10, 120], [100, 50, 20, 0], [-7, 1 << 30, -(1 << 30), 60], [0, 120, 0, 120]):
        x.dev["cu"].copy_(torch.tensor(cu, dtype=torch.int32))
        for max_q in (1, 40, 120):
            il.ilre_paged_attention(x.dev["q"], x.cache(), max_q=max_q, max_kv=1000, out=guard[10:130])
            il.ilre_tree_attention(x.dev["q"], x.cache(), tree, max_q=max_q, max_kv=1000, out=guard[10:130])
        il.ilre_norm_rope_append(x.dev["q"], x.dev["q"][:, :2].contiguous(), None, x.cache(), f, q_out=guard[10:130])
        il.ilre_cache_read(x.cache(), 120, k_out=kv[10:130])
        torch.cuda.synchronize()
        for t in (guard, kv):
            assert (t[:10] == 9).all() and (t[130:] == 9).all()


# ------------------------------------------------------------------------------------------------ trees of drafted tokens

def _tree(q_lens, seed, words=None, blank=()):
    """Random trees: rows of bits, uint32 [T, words]; rows in `blank` see no drafted token, not even themselves."""
    rng = np.random.default_rng(seed)
    words = -(-max(q_lens) // 32) if words is None else words
    rows = []
    for n in q_lens:
        seen = []
        for i in range(n):
            seen.append((seen[rng.integers(max(0, i - 9), i)] if i else 0) | 1 << i)
        rows += seen
    out = np.zeros((len(rows), words), np.uint32)
    for i, r in enumerate(rows):
        for w in range(words):
            out[i, w] = 0 if i in blank else (r >> (32 * w)) & 0xFFFFFFFF
    return out


def _dev(words):
    return torch.from_numpy(words.view(np.int32)).cuda()


def _check_tree(x, words, out, lse):
    row = 0
    for s, (a, n) in enumerate(zip(x.q_lens, x.kv_lens)):
        seen = oq.tree_seen(words[row:row + a], a, n)
        want = oq.attend_seen(_f64(x.q[row:row + a]), _f64(x.k[s]), _f64(x.v[s]), seen)
        _check(out[row:row + a], lse[row:row + a], *want, n, x.dtype, f"sequence {s}: {a} of {n}")
        row += a


TREES = [
    # q_lens, kv_lens, Hq, Hkv, page, layout, dtype
    ([1], [1], 8, 2, 16, "head", "bf16"),
    ([8], [8], 8, 2, 16, "head", "bf16"),                    # nothing but the draft
    ([7, 8, 0, 5], [300, 1031, 9, 5], 32, 8, 64, "head", "bf16"),
    ([8, 8], [4096, 4097], 8, 4, 16, "token", "bf16"),
    ([33, 64], [700, 100], 28, 4, 32, "token", "bf16"),      # a word and a bit; words that straddle tiles
    ([100], [2100], 64, 8, 64, "head", "bf16"),              # 800 rows
    ([130, 3], [131, 3], 8, 2, 16, "head", "bf16"),
    ([12, 6], [5, 2], 8, 2, 16, "head", "bf16"),             # more drafted tokens than the cache holds
    ([8, 3], [500, 3], 8, 2, 32, "head", "f32"),
    ([60], [300], 8, 2, 16, "token", "f32"),
    ([20], [3000], 8, 2, 16, "head", "bf16"),                # 128 rows, cut
    ([64] * 32, [80] * 32, 32, 8, 16, "head", "bf16"),       # 256 rows, whole
    ([4, 3], [3000, 700], 8, 2, 16, "head", "bf16"),         # 16 rows
    ([2], [30], 8, 2, 16, "head", "f32"),
    ([20], [30], 8, 2, 16, "head", "f32"),
    ([5, 9], [2000, 900], 8, 2, 16, "token", "f32"),
]


@pytest.mark.parametrize("fmt", ["plain", "fp8", "fp4"])
@pytest.mark.parametrize("q_lens,kv_lens,Hq,Hkv,page,layout,dtype", TREES)
def test_tree_attention(fmt, q_lens, kv_lens, Hq, Hkv, page, layout, dtype):
    _announce(f"tree {fmt} {q_lens} of {kv_lens} {Hq}/{Hkv} page {page} {layout} {dtype}")
    args = (q_lens, kv_lens, Hq, Hkv, page, dtype, layout)
    x = Paged(*args, seed=sum(kv_lens)) if fmt == "plain" else Quant(fmt, *args, seed=sum(kv_lens))
    limits = dict(max_q=max(q_lens), max_kv=max(kv_lens), total_kv=sum(kv_lens))
    words = _tree(q_lens, sum(q_lens), blank={sum(q_lens) - 1})  # the last one sees the context alone (or nothing at all)
    out, lse = il.ilre_tree_attention(x.dev["q"], x.cache(), _dev(words), **limits)
    torch.cuda.synchronize()
    _check_tree(x, words, out, lse)
    again, lse2 = il.ilre_tree_attention(x.dev["q"], x.cache(), _dev(words), **limits)
    assert torch.equal(out, again) and torch.equal(lse, lse2)
    ws = torch.empty(0, dtype=torch.uint8, device="cuda")
    _check_tree(x, words, *il.ilre_tree_attention(x.dev["q"], x.cache(), _dev(words), workspace=ws, **limits))
    # bits that are nobody's, wider rows, rows with something between them
    wide = np.full((len(words), words.shape[1] + 2), 0xFFFFFFFF, np.uint32)
    wide[:, :words.shape[1]] = words
    row = 0
    for n in q_lens:
        for i in range(n):
            for j in range(n, 32 * words.shape[1]):
                wide[row + i, j // 32] |= np.uint32(1 << (j % 32))
        row += n
    got, lse3 = il.ilre_tree_attention(x.dev["q"], x.cache(), _dev(wide)[:, :words.shape[1]], **limits)
    assert torch.equal(out, got) and torch.equal(lse, lse3)
    got, lse3 = il.ilre_tree_attention(x.dev["q"], x.cache(), _dev(wide), **limits)
    assert torch.equal(out, got) and torch.equal(lse, lse3)


@pytest.mark.parametrize("fmt", ["plain", "fp8", "fp4"])
@pytest.mark.parametrize("q_lens,kv_lens,Hq,Hkv,page,layout,dtype", TREES)
def test_drafted_tokens_that_nobody_sees_hold_anything(fmt, q_lens, kv_lens, Hq, Hkv, page, layout, dtype):
    """Drafted tokens that were given up, or never filled in, between others that are seen."""
    _announce(f"tree, unseen drafts, {fmt} {q_lens} of {kv_lens} {Hq}/{Hkv} page {page} {layout} {dtype}")
    args = (q_lens, kv_lens, Hq, Hkv, page, dtype, layout)
    x = Paged(*args, seed=sum(kv_lens)) if fmt == "plain" else Quant(fmt, *args, seed=sum(kv_lens))
    words = _tree(q_lens, sum(q_lens))
    row = 0
    for s, (n, kv) in enumerate(zip(q_lens, kv_lens)):
        for j in range(1, n, 3):
            words[row:row + n, j // 32] &= np.uint32(~(1 << (j % 32)) & 0xFFFFFFFF)
            at = kv - n + j
            if at < 0:
                continue
            where = (int(x.table[s, at // page]), slice(None), at % page)
            for p in (x.kp, x.vp):
                if fmt == "plain":
                    p[where] = float("nan") if j % 2 else float("inf")
                else:
                    p.view(torch.uint8)[where] = 0x7F
            if fmt != "plain":
                x.ks[where] = x.vs[where] = 255
        row += n
    out, lse = il.ilre_tree_attention(x.dev["q"], x.cache(), _dev(words), max_q=max(q_lens), max_kv=max(kv_lens), total_kv=sum(kv_lens))
    torch.cuda.synchronize()
    _check_tree(x, words, out, lse)


@pytest.mark.parametrize("fmt,dtype", [("plain", "bf16"), ("plain", "f32"), ("fp8", "bf16"), ("fp4", "bf16")])
def test_drafts_over_contexts_promised_long(fmt, dtype):
    """(Cut up, and read, as if the contexts were far longer than they are.)"""
    _announce(f"tree, long contexts promised, {fmt} {dtype}")
    q_lens, kv_lens = [7, 8, 0, 5], [300, 1031, 9, 5]
    args = (q_lens, kv_lens, 32, 8, 64, dtype, "token")
    x = Paged(*args, seed=8) if fmt == "plain" else Quant(fmt, *args, seed=8)
    words = _tree(q_lens, 8, blank={3})
    run = lambda **kw: il.ilre_tree_attention(x.dev["q"], x.cache(), _dev(words), max_q=8, max_kv=400000, total_kv=800000, **kw)  # noqa: E731
    out, lse = run()
    torch.cuda.synchronize()
    _check_tree(x, words, out, lse)
    again, lse2 = run()
    assert torch.equal(out, again) and torch.equal(lse, lse2)
    _check_tree(x, words, *run(workspace=torch.empty(0, dtype=torch.uint8, device="cuda")))


def test_more_drafted_tokens_than_bits():
    """A sequence longer than max_q promised: what has no bit is not seen."""
    _announce("tree, too few words")
    x = Paged([50], [400], 8, 2, 16, "bf16", seed=4)
    words = _tree([50], 4)[:, :1]
    _check_tree(x, words, *il.ilre_tree_attention(x.dev["q"], x.cache(), _dev(words), max_q=32, max_kv=400))


def test_a_chain_is_causal_attention():
    _announce("tree, chain")
    for q_lens, kv_lens in (([8, 5], [900, 40]), ([70], [1000])):
        x = Paged(q_lens, kv_lens, 8, 2, 16, "bf16", seed=11)
        words = np.concatenate([[[(((1 << (i + 1)) - 1) >> (32 * w)) & 0xFFFFFFFF for w in range(3)] for i in range(n)] for n in q_lens]).astype(np.uint32)
        out, lse = il.ilre_tree_attention(x.dev["q"], x.cache(), _dev(words), max_q=max(q_lens), max_kv=max(kv_lens))
        x.check(out, lse)


def test_absent_pages_under_a_tree():
    _announce("tree, absent pages")
    for fmt in ("plain", "fp8"):
        for n in (6, 40):
            args = ([n], [500], 8, 2, 16, "bf16")
            x = Paged(*args, seed=12) if fmt == "plain" else Quant(fmt, *args, seed=12)
            words = _tree([n], 12)
            gone = np.zeros(500, bool)
            for col in (0, 9, 31):  # the last one holds drafted tokens
                x.dev["table"][0, col] = -1
                gone[col * 16:col * 16 + 16] = True
            out, lse = il.ilre_tree_attention(x.dev["q"], x.cache(), _dev(words), max_q=n, max_kv=500)
            want = oq.attend_seen(_f64(x.q), _f64(x.k[0]), _f64(x.v[0]), oq.tree_seen(words, n, 500) & ~gone)
            _check(out, lse, *want, 500, "bf16")


# ------------------------------------------------------------------------------------------------ filling a cache

def _weights(dtype, seed, offset):
    g = torch.Generator().manual_seed(seed)
    return [(torch.randn(128, generator=g) * 0.3 + 1 - offset).to(DT[dtype]) for _ in range(2)]


def _states(T, Hq, Hkv, dtype, seed):
    """Queries, keys and values side by side in one row, with blocks that a quantiser has to look at: zeros, small and large ones."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(T, Hq + 2 * Hkv, 128, generator=g) * torch.exp(2 * torch.randn(T, Hq + 2 * Hkv, 1, generator=g))
    x[0, -1, :32] = 0
    x[0, -1, 32:64] *= 1e-37
    x[0, -1, 64:96] *= 1e30
    return x.to(DT[dtype])


FILLS = [
    # dtype, fmt, layout, pairing, rotary, axes, norm, offset, page
    ("bf16", "fp8", "head", "half", 128, 1, "both", 0, 16),
    ("bf16", "fp4", "token", "half", 128, 3, "both", 1, 32),
    ("bf16", "fp8", "token", "half", 64, 3, "k", 0, 16),
    ("bf16", "fp4", "head", "half", 96, 1, "both", 0, 64),
    ("bf16", "fp8", "head", "interleaved", 64, 3, "both", 0, 16),
    ("bf16", "fp8", "head", "half", 16, 1, "none", 0, 16),
    ("bf16", "fp4", "head", "interleaved", 128, 1, "none", 0, 16),
    ("bf16", "fp8", "head", "half", 0, 1, "both", 0, 16),
    ("bf16", "plain", "head", "half", 128, 3, "both", 0, 16),
    ("bf16", "plain", "token", "half", 96, 1, "both", 1, 32),
    ("bf16", "plain", "head", "interleaved", 64, 3, "q", 0, 16),
    ("f32", "fp8", "token", "half", 128, 1, "both", 0, 16),
    ("f32", "fp4", "head", "half", 64, 3, "both", 1, 16),
    ("f32", "fp8", "head", "interleaved", 96, 1, "none", 0, 32),
    ("f32", "plain", "token", "half", 128, 3, "both", 0, 16),
    ("f32", "plain", "head", "interleaved", 16, 1, "both", 1, 16),
    ("f32", "plain", "head", "half", 0, 1, "q", 0, 16),
]


def _turned(x, weight, positions, axes, f, pairing, offset):
    """fp64: x normed (weight None: not) and turned."""
    y = _f64(x) if weight is None else oq.norm(_f64(x), _f64(weight), 1e-6, offset)
    return y if f is None else oq.rope_axes(y, positions, axes, np.array(f.inv_freq)[:f.rotary // 2], f.magnitude, pairing)


def _near(got, want, size, dtype):
    """Sines and cosines are off by 2^-23, the products and sums of a pair and its norm by 2^-24 each, a dozen of them: 2^-20 of the pair's size together, before the last rounding."""
    tol = HALF[dtype] * 1.001 * np.abs(want) + 2.0 ** -20 * size + 2.0 ** -140
    err = np.abs(_f64(got) - want)
    assert (err <= tol).all(), float((err / tol).max())


@pytest.mark.parametrize("q_lens,kv_lens", [([1, 1, 1], [1, 700, 64]), ([1, 0, 40, 3], [700, 5, 40, 64]), ([4200], [4300])], ids=["steps", "chunks", "many"])
@pytest.mark.parametrize("dtype,fmt,layout,pairing,rotary,axes,norm,offset,page", FILLS)
def test_fill(dtype, fmt, layout, pairing, rotary, axes, norm, offset, page, q_lens, kv_lens):
    _announce(f"fill {q_lens} {dtype} {fmt} {layout} {pairing} {rotary} axes {axes} norm {norm} offset {offset} page {page}")
    T, Hq, Hkv, S = sum(q_lens), 6, 2, len(q_lens)
    args = (q_lens, kv_lens, Hq, Hkv, page, dtype, layout)
    x = Paged(*args, fill=0.5) if fmt == "plain" else Quant(fmt, *args)
    fused = _states(T, Hq, Hkv, dtype, T + rotary)
    q, k, v = fused[:, :Hq], fused[:, Hq:Hq + Hkv], fused[:, Hq + Hkv:]
    qw, kw = _weights(dtype, rotary, offset)
    qw, kw = (qw if norm in ("both", "q") else None), (kw if norm in ("both", "k") else None)
    f = il.ilre_rope_frequencies(rotary, BASE, scaling=il.ILRE_ROPE_PARTS, factor=8.0, low=1.0, high=32.0, original_len=4096) if rotary else None
    places = np.concatenate([np.arange(n - a, n) for a, n in zip(q_lens, kv_lens)])
    pos = places[None] if axes == 1 else np.stack((places, places // 7 - 20, places % 31 + 5))
    table = (0,) * (rotary // 2) if axes == 1 else AXES3[rotary // 2]
    x.dev["table"][S - 1, x.dev["table"].shape[1] - 1] = -1 if S == 4 else x.dev["table"][S - 1, -1]
    before = {n: getattr(x, n).clone() for n in ("kp", "vp") + (("ks", "vs") if fmt != "plain" else ())}
    dev = fused.cuda()
    norms = None if norm == "none" else il.HeadNorms(None if qw is None else qw.cuda(), None if kw is None else kw.cuda(), eps=1e-6, offset=offset)
    got = il.ilre_norm_rope_append(dev[:, :Hq], dev[:, Hq:Hq + Hkv], dev[:, Hq + Hkv:], x.cache(), f, None if axes == 1 else torch.from_numpy(pos).int().cuda(),
                                   norms=norms, axes=None if axes == 1 else table, pairing=il.ILRE_ROPE_HALF if pairing == "half" else il.ILRE_ROPE_INTERLEAVED)
    torch.cuda.synchronize()
    want_q, want_k = (_turned(t, w, pos, table, f, pairing, offset) for t, w in ((q, qw), (k, kw)))
    for t, w, want, name in ((q, qw, want_q, "q"), (k, kw, want_k, "k")):
        size = np.abs(_f64(t) if w is None else oq.norm(_f64(t), _f64(w), 1e-6, offset)).max(-1, keepdims=True) * (2 * f.magnitude if f else 1)
        if name == "q":
            _near(got, want, size, dtype)
        else:
            k_size = size
    seq = np.repeat(np.arange(S), q_lens)
    dev_table = x.dev["table"].cpu()
    stored = torch.from_numpy(np.array([int(dev_table[s, p // page]) >= 0 for s, p in zip(seq, places)], dtype=bool))
    page_at, cell = dev_table[seq, places // page].long()[stored].cuda(), torch.from_numpy(places % page)[stored].cuda()
    if fmt == "plain":
        _near(x.kp[page_at, :, cell], want_k[stored.numpy()], k_size[stored.numpy()], dtype)
        assert torch.equal(x.vp[page_at, :, cell].cpu(), v[stored])
    else:
        for pages, scales, want in ((x.kp, x.ks, want_k), (x.vp, x.vs, _f64(v))):
            codes, sc = oq.store(want[stored.numpy()], fmt)
            assert np.array_equal(scales[page_at, :, cell].cpu().numpy(), sc)
            mine = _u8(pages)[page_at.cpu(), :, cell.cpu()]
            assert np.array_equal(mine, codes), (int((mine != codes).sum()), mine.size)
    for name, old in before.items():  # nothing else was touched
        new = getattr(x, name)
        u = (lambda t: t.view(torch.uint8)) if name in ("kp", "vp") and fmt == "fp8" else (lambda t: t)
        u(old)[page_at, :, cell] = u(new)[page_at, :, cell]
        assert torch.equal(u(old), u(new)), name


def test_rope_append_takes_a_quantised_cache():
    _announce("rope_append, quantised")
    for fmt in ("fp8", "fp4"):
        x, y = (Quant(fmt, [5, 60], [100, 60], 8, 2, 16, "bf16", seed=2) for _ in range(2))
        s = _states(65, 8, 2, "bf16", 3).cuda()
        f = il.ilre_rope_frequencies(64, BASE)
        a = il.ilre_rope_append(s[:, :8], s[:, 8:10], s[:, 10:], x.cache(), f)
        b = il.ilre_norm_rope_append(s[:, :8], s[:, 8:10], s[:, 10:], y.cache(), f)
        assert torch.equal(a, b) and torch.equal(x.ks, y.ks) and torch.equal(x.vs, y.vs)
        assert np.array_equal(_u8(x.kp), _u8(y.kp)) and np.array_equal(_u8(x.vp), _u8(y.vp))


@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
def test_infinities_and_nan_mark_their_block(fmt):
    _announce(f"fill, infinities and NaN {fmt}")
    x = Quant(fmt, [3], [40], 8, 2, 16, "f32", seed=2)
    v = torch.randn(3, 2, 128)
    v[0, 0, 3], v[1, 1, 40], v[2, 0, 127] = float("inf"), float("nan"), -float("inf")
    v[2, 1, 64:96] = 3.4028234663852886e38
    il.ilre_norm_rope_append(None, v.cuda(), v.cuda(), x.cache(), None)
    k_out, v_out = il.ilre_cache_read(x.cache(), 3, dtype=torch.float32)
    codes, scales = oq.store(_f64(v), fmt)
    want = oq.read(codes, scales, fmt)
    assert want[2, 1, 64] == 2.0 ** 128  # the largest float is 2^128 (1 - 2^-24): the nearest code under its scale is 2^128, which fp32 rounds to an infinity
    with np.errstate(over="ignore"):
        want = want.astype(np.float32).astype(np.float64)
    for got in (k_out, v_out):
        same = np.array_equal(_f64(got), want, equal_nan=True)
        assert same and np.isnan(want).sum() == 96
    t = np.arange(37, 40)
    assert np.array_equal(x.vs[x.table[0, t // 16].long(), :, t % 16].cpu().numpy(), scales)


def test_norm_rope_alone():
    _announce("norm_rope")
    for dtype in ("bf16", "f32"):
        for T, H, rotary in ((1, 1, 128), (77, 5, 64), (5000, 2, 128)):
            g = torch.Generator().manual_seed(T)
            x = torch.randn(T, H, 128, generator=g).to(DT[dtype])
            w = _weights(dtype, T, 0)[0]
            f = il.ilre_rope_frequencies(rotary, BASE)
            pos = torch.randint(-1000, 100000, (T,), generator=g).int()
            size = np.abs(oq.norm(_f64(x), _f64(w), 1e-6)).max(-1, keepdims=True) * 2
            got = il.ilre_norm_rope(x.cuda(), f, pos.cuda(), norms=il.HeadNorms(w.cuda()))
            _near(got, _turned(x, w, pos.numpy()[None], [0] * (rotary // 2), f, "half", 0), size, dtype)
            y = x.cuda()
            assert il.ilre_norm_rope(y, f, pos.cuda(), norms=il.HeadNorms(w.cuda()), out=y) is y and torch.equal(y, got)
            got = il.ilre_norm_rope(x.cuda(), f, first_position=77)
            _rope_check(got, x, 77 + np.arange(T), f, "half", dtype, rotary)
            got = il.ilre_norm_rope(x.cuda(), None)
            assert torch.equal(got.cpu(), x)
    assert il.ilre_norm_rope(torch.empty(0, 2, 128, device="cuda"), None).shape == (0, 2, 128)


def test_fill_leaves_out_what_has_no_place():
    _announce("fill, no place")
    f = il.ilre_rope_frequencies(128, BASE)
    for kv in (5, 1000, -3):  # 20 new tokens end at 5: 15 lie in front of the cache; at 1000: behind the table of 4 pages
        x = Quant("fp8", [20], [64], 4, 2, 16, "bf16", seed=1)
        x.dev["kv_len"].fill_(kv)
        before = _u8(x.vp), x.vs.cpu().numpy()
        s = _states(20, 4, 2, "bf16", 5)
        got = il.ilre_norm_rope_append(s.cuda()[:, :4], s.cuda()[:, 4:6], s.cuda()[:, 6:], x.cache(), f)
        _near(got, _turned(s[:, :4], None, (kv - 20 + np.arange(20))[None], [0] * 64, f, "half", 0), np.abs(_f64(s[:, :4])).max(-1, keepdims=True) * 2, "bf16")
        codes, scales = oq.store(_f64(s[15:, 6:]), "fp8")
        if kv == 5:
            at = int(x.table[0, 0])
            before[0][at, :, :5], before[1][at, :, :5] = codes.transpose(1, 0, 2), scales.transpose(1, 0, 2)
        assert np.array_equal(_u8(x.vp), before[0]) and np.array_equal(x.vs.cpu().numpy(), before[1])


# ------------------------------------------------------------------------------------------------ reading back

@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_every_code_under_every_scale(fmt, dtype):
    _announce(f"read, all codes {fmt} {dtype}")
    n = 256  # token t has scale byte t (and others); its codes run through all of them
    codes = np.stack([np.arange(t, t + (128 if fmt == "fp8" else 64)) % 256 for t in range(n)]).astype(np.uint8)[:, None]
    codes = np.concatenate([codes, codes ^ 128], 1)  # two kv heads
    scales = np.stack([(t + 64 * np.arange(4)) % 256 for t in range(n)]).astype(np.uint8)[:, None].repeat(2, 1)
    scales = np.maximum(scales, 1)
    pages = torch.from_numpy(codes.reshape(16, 16, 2, -1).transpose(0, 2, 1, 3).copy()).cuda()
    sc = torch.from_numpy(scales.reshape(16, 16, 2, 4).transpose(0, 2, 1, 3).copy()).cuda()
    pages = pages.view(torch.float8_e4m3fn) if fmt == "fp8" else pages
    cache = il.QuantKV(pages, None, sc, None, torch.arange(16, dtype=torch.int32, device="cuda")[None], _i32(n), _i32(0, n))
    k, none = il.ilre_cache_read(cache, n, dtype=DT[dtype])
    assert none is None
    want = torch.from_numpy(oq.read(codes, scales, fmt))
    want = want.float().to(DT[dtype])  # (exact, but for those below 2^-133 in bf16, rounded, and those past the type's largest)
    assert torch.equal(k.cpu().nan_to_num(7.5), want.nan_to_num(7.5))


@pytest.mark.parametrize("fmt,dtype", [("fp8", "bf16"), ("fp4", "bf16"), ("fp8", "f32"), ("plain", "bf16"), ("plain", "f32")])
@pytest.mark.parametrize("layout", ["head", "token"])
def test_read(fmt, dtype, layout):
    _announce(f"read {fmt} {dtype} {layout}")
    lens = [300, 1, 0, 777, 64]
    args = ([0] * 5, lens, 4, 2, 32, dtype, layout)
    x = Paged(*args, seed=3) if fmt == "plain" else Quant(fmt, *args, seed=3)
    x.dev["table"][3, 2] = -1  # tokens 64 .. 95 of the fourth sequence are on no page
    k, v = [[t.double() for t in s] for s in (x.k, x.v)]
    for t in (k, v):
        t[3][64:96] = 0

    def want(tokens):  # by sequence
        return [torch.cat([torch.stack([t[s][i] if 0 <= i < lens[s] else torch.zeros(2, 128, dtype=torch.double) for i in ts]) if len(ts) else torch.zeros(0, 2, 128, dtype=torch.double)
                           for s, ts in enumerate(tokens)]) for t in (k, v)]

    # whole sequences; the last tokens of each; more than there are (zeros in front)
    for rows in (lens, [min(n, 40) for n in lens], [n + 3 for n in lens]):
        x.dev["cu"].copy_(torch.tensor([0] + list(np.cumsum(rows)), dtype=torch.int32))
        T = sum(rows)
        got = il.ilre_cache_read(x.cache(), T, dtype=DT[dtype])
        for a, b in zip(got, want([range(n - r, n) for n, r in zip(lens, rows)])):
            assert torch.equal(a.cpu().double(), b)
    # some tokens, in no order, some twice, some that are not there; into the recall's layout, and rows of no sequence
    rng = np.random.default_rng(0)
    tokens = [rng.integers(-3, n + 5, r).tolist() for n, r in zip(lens, (50, 3, 4, 500, 0))]
    flat = [t for ts in tokens for t in ts]
    x.dev["cu"].copy_(torch.tensor([2] + list(2 + np.cumsum([len(t) for t in tokens])), dtype=torch.int32))
    T = len(flat) + 5
    out = [torch.full((2, T, 128), 9.0, dtype=DT[dtype], device="cuda") for _ in range(2)]
    il.ilre_cache_read(x.cache(), T, _i32(0, 0, *flat, 0, 0, 0), k_out=out[0].transpose(0, 1), v_out=out[1].transpose(0, 1))
    for a, b in zip(out, want(tokens)):
        a = a.transpose(0, 1).cpu()
        assert torch.equal(a[2:-3].double(), b) and (a[:2] == 9).all() and (a[-3:] == 9).all()
    # values alone, in wider rows
    wide = torch.full((T, 5, 128), 9.0, dtype=DT[dtype], device="cuda")
    assert il.ilre_cache_read(x.cache(), T, _i32(0, 0, *flat, 0, 0, 0), v_out=wide[:, 1:3])[0] is None
    assert torch.equal(wide[2:-3, 1:3].cpu().double(), want(tokens)[1]) and (wide[:, 3:] == 9).all() and (wide[:, 0] == 9).all()
    assert il.ilre_cache_read(x.cache(), 0)[0].shape == (0, 2, 128)


def test_reading_for_many_sequences():
    _announce("read, 300 sequences")
    lens = [i % 5 for i in range(300)]
    x = Quant("fp8", [0] * 300, lens, 4, 2, 16, "bf16", seed=1)
    x.dev["cu"].copy_(torch.tensor([0] + list(np.cumsum(lens)), dtype=torch.int32))
    T = sum(lens)
    want = torch.cat(x.k)
    assert torch.equal(il.ilre_cache_read(x.cache(), T)[0].cpu().double(), want)
    out = torch.empty(2, T, 128, dtype=torch.bfloat16, device="cuda")
    il.ilre_cache_read(x.cache(), T, k_out=out.transpose(0, 1))
    assert torch.equal(out.transpose(0, 1).cpu().double(), want)


# ------------------------------------------------------------------------------------------------ together

def test_strides_streams_and_tokens_of_no_sequence():
    _announce("quantised, strided q and out, another stream, tokens of no sequence")
    x = Quant("fp8", [5, 40], [300, 41], 8, 2, 32, "bf16", seed=8)
    T = 45
    wide = torch.randn(T + 6, 12, 128, device="cuda").bfloat16()
    wide[3:3 + T, 2:10] = x.dev["q"]
    x.dev["cu"] += 3
    words = np.zeros((T + 6, 2), np.uint32)
    words[3:3 + T] = _tree([5, 40], 1)
    tree = _dev(words)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    for call in ("paged", "tree"):
        outs = torch.full((T + 6, 9, 256), 7.0, device="cuda").bfloat16()
        lse = torch.full((T + 6, 8), 7.0, device="cuda")
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            kw = dict(max_q=40, max_kv=300, out=outs[:, :8, 128:], lse=lse)
            out, _ = il.ilre_paged_attention(wide[:, 2:10], x.cache(), **kw) if call == "paged" else il.ilre_tree_attention(wide[:, 2:10], x.cache(), tree, **kw)
        stream.synchronize()
        assert (outs[:, 8] == 7).all() and (outs[..., :128] == 7).all() and (outs[:3] == 7).all() and (outs[3 + T:] == 7).all()
        assert (lse[:3] == 7).all() and (lse[3 + T:] == 7).all()
        if call == "paged":
            x.check(out[3:3 + T], lse[3:3 + T])
        else:
            _check_tree(x, words[3:3 + T], out[3:3 + T], lse[3:3 + T])


def test_captured_steps_follow_what_is_written_later():
    """Fill, attention and a drafted tree in one graph; each replay against the eager calls."""
    _announce("quantised, graph")
    x = Quant("fp8", [2, 2, 2], [700, 33, 2000], 8, 2, 16, "bf16", seed=9)
    cache, s = x.cache(), _states(6, 8, 2, "bf16", 9).cuda()
    f, norms = il.ilre_rope_frequencies(128, BASE), il.HeadNorms(*(w.cuda() for w in _weights("bf16", 1, 0)))
    tree = _dev(_tree([2, 2, 2], 3))
    ws = [il.alloc_workspace_attention(6, 3, 8, 2, 128, 2, 2000) for _ in range(2)]
    q = torch.empty(6, 8, 128, dtype=torch.bfloat16, device="cuda")
    outs, lses = [torch.empty_like(q) for _ in range(2)], [torch.empty(6, 8, device="cuda") for _ in range(2)]
    back = [torch.empty(6, 2, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2)]

    def run():
        il.ilre_norm_rope_append(s[:, :8], s[:, 8:10], s[:, 10:], cache, f, norms=norms, q_out=q)
        il.ilre_paged_attention(q, cache, max_q=2, max_kv=2000, workspace=ws[0], out=outs[0], lse=lses[0])
        il.ilre_tree_attention(q, cache, tree, max_q=2, max_kv=2000, workspace=ws[1], out=outs[1], lse=lses[1])
        il.ilre_cache_read(cache, 6, k_out=back[0], v_out=back[1])

    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for lens in ([700, 33, 2000], [2, 30, 1999], [350, 3, 16], [700, 33, 2000]):
        x.dev["kv_len"].copy_(torch.tensor(lens, dtype=torch.int32))
        s.copy_(_states(6, 8, 2, "bf16", sum(lens)))
        for t in (q, *outs, *lses, *back):
            t.fill_(5.0)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (q, *outs, *lses, *back)]
        run()
        torch.cuda.synchronize()
        for a, b in zip(got, (q, *outs, *lses, *back)):
            assert torch.equal(a, b)
        for a in (0, 1):
            assert np.isfinite(_f64(outs[a])).all()


def test_pools_beyond_32_bits():
    """Pages at both ends of pools of 5 GiB of codes."""
    _announce("quantised, pool of 5 GiB")
    for fmt, pages in (("fp8", 82000), ("fp4", 164000)):
        code = torch.zeros(pages, 8, 64, 128 if fmt == "fp8" else 64, dtype=torch.uint8, device="cuda")
        scale = torch.zeros(pages, 8, 64, 4, dtype=torch.uint8, device="cuda")
        kp = code.view(torch.float8_e4m3fn) if fmt == "fp8" else code
        n, used = 64 * 5, [0, pages - 1, 40000, pages - 2, 65536]
        cache = il.QuantKV(kp, kp, scale, scale, _i32(*used)[None], _i32(n), _i32(0, n))
        g = torch.Generator().manual_seed(10)
        k, q = torch.randn(n, 8, 128, generator=g).bfloat16(), torch.randn(3, 32, 128, generator=g).bfloat16()
        il.ilre_norm_rope_append(None, k.cuda(), k.cuda(), cache, None)
        stored = oq.store(_f64(k), fmt)
        value = oq.read(*stored, fmt)
        for i, p in enumerate(used):
            assert np.array_equal(code[p].cpu().numpy().transpose(1, 0, 2), stored[0][i * 64:i * 64 + 64])
        assert np.array_equal(_f64(il.ilre_cache_read(cache, n)[1]), value)
        cache = il.QuantKV(kp, kp, scale, scale, _i32(*used)[None], _i32(n), _i32(0, 3))
        out, lse = il.ilre_paged_attention(q.cuda(), cache, max_q=3, max_kv=n)
        _check(out, lse, *oa.attend(_f64(q), value, value), n, "bf16")
        del code, scale, kp, cache


def test_nothing_to_do():
    _announce("quantised, nothing to do")
    x = Quant("fp8", [0, 0], [5, 0], 8, 2, 16, "bf16")
    e = torch.empty(0, 2, 128, dtype=torch.bfloat16, device="cuda")
    out, lse = il.ilre_paged_attention(x.dev["q"], x.cache(), max_q=0, max_kv=5)
    assert out.shape == (0, 8, 128) and lse.shape == (0, 8)
    assert il.ilre_tree_attention(x.dev["q"], x.cache(), torch.empty(0, 1, dtype=torch.int32, device="cuda"), max_q=0, max_kv=5)[0].shape == (0, 8, 128)
    assert il.ilre_norm_rope_append(x.dev["q"], e, e, x.cache(), None).shape == (0, 8, 128)


def test_another_device_is_refused():
    """(One GPU here: a tensor that says it is elsewhere.)"""
    class Elsewhere(torch.Tensor):
        def get_device(self):
            return 1

    x = Quant("fp8", [1], [5], 8, 2, 16, "bf16")
    q = x.dev["q"].as_subclass(Elsewhere)
    with pytest.raises(ValueError, match="device"):
        il.ilre_tree_attention(q, x.cache(), _i32(1)[None], max_q=1, max_kv=5)
    with pytest.raises(il.IlreError):
        il.ilre_tree_attention(x.dev["q"], x.cache(), _i32(1)[None], max_q=33, max_kv=5)
    with pytest.raises(ValueError, match="device"):
        il.ilre_norm_rope(x.dev["q"], None, norms=il.HeadNorms(torch.ones(128, dtype=torch.bfloat16, device="cuda").as_subclass(Elsewhere)))
    for name in ("ks", "vs", "vp"):
        x = Quant("fp8", [1], [5], 8, 2, 16, "bf16")
        setattr(x, name, getattr(x, name).as_subclass(Elsewhere))
        with pytest.raises(ValueError, match="device"):
            x.cache()


def test_a_request_over_a_quantised_cache():
    """Chunks of a context are normed, turned along three axes, stored in 8 bits and attended to; the keys are read back for the recall, the kept tokens stored in 4 bits, and a draft attends
    to them: every stage against the oracle on what the stage before should have left."""
    _announce("a request, every operator")
    L, HQ, HKV, P = 620, 8, 2, 16
    g = torch.Generator().manual_seed(31)
    states = torch.randn(L, HQ + 2 * HKV, 128, generator=g).bfloat16()
    qw, kw = _weights("bf16", 31, 0)
    f = il.ilre_rope_frequencies(128, 500000.0)
    pos = np.stack((np.arange(L), np.arange(L) // 7, np.arange(L) % 7))
    pages = -(-L // P)
    blank = lambda width: torch.full((pages + 1, HKV, P, width), 255, dtype=torch.uint8, device="cuda")  # noqa: E731
    kp, vp, ks, vs = blank(128).view(torch.float8_e4m3fn), blank(128).view(torch.float8_e4m3fn), blank(4), blank(4)
    table = torch.randperm(pages + 1, generator=g)[:pages].int().cuda()[None]
    kv_len, cu = _i32(0), _i32(0, 0)
    cache = il.QuantKV(kp, vp, ks, vs, table, kv_len, cu)
    norms = il.HeadNorms(qw.cuda(), kw.cuda())
    dev = states.cuda()
    want_k = oq.read(*oq.store(_turned(states[:, HQ:HQ + HKV], kw, pos, AXES3[64], f, "half", 0), "fp8"), "fp8")
    want_v = oq.read(*oq.store(_f64(states[:, HQ + HKV:]), "fp8"), "fp8")
    at = 0
    for n in (204, 200, 200, 16):
        s = dev[at:at + n]
        kv_len.fill_(at + n)
        cu[1] = n
        q = il.ilre_norm_rope_append(s[:, :HQ], s[:, HQ:HQ + HKV], s[:, HQ + HKV:], cache, f, torch.from_numpy(pos[:, at:at + n].copy()).int().cuda(), norms=norms, axes=AXES3[64])
        out, lse = il.ilre_paged_attention(q, cache, max_q=n, max_kv=at + n, sink=4, window=128)
        _check(out, lse, *oa.attend(_f64(q), want_k[:at + n], want_v[:at + n], sink=4, window=128), at + n, "bf16", f"chunk at {at}")
        at += n
    # the last chunk's queries recall, over the keys as they come out of the cache
    cu[1] = L
    key_cache = torch.empty(HKV, L, 128, dtype=torch.bfloat16, device="cuda")
    il.ilre_cache_read(cache, L, k_out=key_cache.transpose(0, 1))
    assert np.array_equal(_f64(key_cache.transpose(0, 1)), want_k)
    idx, _ = il.ilre_recall(q.transpose(0, 1), key_cache, 90, (1, 3, 7), sink=4)
    assert len(idx) == 94
    cu[1] = len(idx)
    k, v = il.ilre_cache_read(cache, len(idx), idx)
    kept = idx.cpu().numpy()
    assert np.array_equal(_f64(k), want_k[kept]) and np.array_equal(_f64(v), want_v[kept])
    # kept tokens and a draft of six in 4 bits (the keys are turned already)
    n, m = 6, len(idx) + 6
    k, v = torch.cat((k, dev[:n, HQ:HQ + HKV])), torch.cat((v, dev[:n, HQ + HKV:]))
    code, scale = torch.zeros(8, HKV, P, 64, dtype=torch.uint8, device="cuda"), torch.zeros(8, HKV, P, 4, dtype=torch.uint8, device="cuda")
    code2, scale2 = torch.zeros_like(code), torch.zeros_like(scale)
    short = il.QuantKV(code, code2, scale, scale2, _i32(6, 1, 4, 2, 7, 0, 3)[None], _i32(m), _i32(0, m))
    il.ilre_norm_rope_append(None, k, v, short, None)
    short.cu_q[1] = n
    words = _tree([n], 5)
    out, lse = il.ilre_tree_attention(q[:n].contiguous(), short, _dev(words), max_q=n, max_kv=m)
    k4, v4 = (oq.read(*oq.store(_f64(t), "fp4"), "fp4") for t in (k, v))
    _check(out, lse, *oq.attend_seen(_f64(q[:n]), k4, v4, oq.tree_seen(words, n, m)), m, "bf16", "draft")
