"""GPU parity of the operators around a recall, through the C ABI, against the fp64 oracle on the same inputs.

Tolerances, from the arithmetic.  A row's logits are fp32 sums of 128 exact products (bf16) or rounded ones (fp32): off by at most 130 * 2^-24 times the sum of
their magnitudes, `reach`.  Weights exp2(fma(s, c, -m)) add 2^-23 per unit of the exponent, at most 2 reach + 64 units here, and 2^-22 of the exponential itself.
Sums of n weights are at most n / 8 + 16 additions deep.  With bf16 states a weight is rounded once more, by 2^-8 of itself at most, before the product with V.
So |out - exact| <= eps_out |exact| + (2 eps_w + eps_p) sum_t p |v|, |lse - exact| <= eps_w + 2^-22 |exact|.
"""
import numpy as np
import pytest
import torch

import paper_2508_17892_amd as il
from oracle import attention as oa

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


def _announce(msg):
    print(f"[case] {msg}", flush=True)


def _f64(t):
    return t.detach().double().cpu().numpy()


def _check(got, lse, want, want_lse, size, reach, n, dtype, what=""):
    eps_w = 130 * 2.0 ** -24 * reach + (2 * reach + 64) * 2.0 ** -23 + 2.0 ** -22 + (n / 8 + 16) * 2.0 ** -24
    eps_p = HALF["bf16"] if dtype == "bf16" else 0.0
    tol = HALF[dtype] * 1.01 * np.abs(want) + ((2 * eps_w + eps_p)[..., None] * size) + 1e-30
    got, lse = _f64(got), _f64(lse)
    assert np.isfinite(got).all(), what
    err = np.abs(got - want)
    assert (err <= tol).all(), (what, float((err / tol).max()), np.argwhere(err > tol)[:3].tolist())
    none = np.isinf(want_lse)
    assert (lse[none] == -np.inf).all() and (got[none] == 0).all(), what
    d = np.abs(np.subtract(lse, want_lse, where=~none, out=np.zeros_like(want_lse)))
    assert (d <= eps_w + 2.0 ** -22 * np.abs(np.where(none, 0, want_lse))).all(), (what, float(d.max()))


class Paged:
    """Random sequences in pages of no order.  `fill`: what everything that is nobody's token holds."""

    def __init__(self, q_lens, kv_lens, Hq, Hkv, page, dtype, layout="head", seed=0, fill=float("nan"), spare=2, width=None, scale=1.0):
        g = torch.Generator().manual_seed(seed)
        self.q_lens, self.kv_lens, self.dtype, self.page = q_lens, kv_lens, dtype, page
        need = [-(-n // page) for n in kv_lens]
        total = sum(need) + spare
        shape = (total, page, Hkv, 128) if layout == "token" else (total, Hkv, page, 128)
        self.pages = [torch.full(shape, fill, dtype=DT[dtype]) for _ in range(2)]
        view = [p.permute(0, 2, 1, 3) if layout == "token" else p for p in self.pages]
        order = torch.randperm(total, generator=g)
        width = max(max(need, default=1), 1) if width is None else width
        table = torch.full((len(kv_lens), width), -7, dtype=torch.int32)
        self.q = (torch.randn(sum(q_lens), Hq, 128, generator=g) * scale).to(DT[dtype])
        self.k, self.v = [], []
        at = 0
        for s, n in enumerate(kv_lens):
            table[s, :need[s]] = order[at:at + need[s]].int()
            at += need[s]
            k, v = torch.randn(n, Hkv, 128, generator=g).to(DT[dtype]), torch.randn(n, Hkv, 128, generator=g).to(DT[dtype])
            for t in range(0, n, page):
                m = min(page, n - t)
                view[0][table[s, t // page], :, :m] = k[t:t + m].transpose(0, 1)
                view[1][table[s, t // page], :, :m] = v[t:t + m].transpose(0, 1)
            self.k.append(k)
            self.v.append(v)
        self.table = table
        self.kp, self.vp = (v.to("cuda") if layout == "head" else p.to("cuda").permute(0, 2, 1, 3) for v, p in zip(view, self.pages))
        self.dev = dict(q=self.q.cuda(), table=table.cuda(), kv_len=torch.tensor(kv_lens, dtype=torch.int32).cuda(),
                        cu=torch.tensor([0] + list(np.cumsum(q_lens)), dtype=torch.int32).cuda())

    def cache(self):
        return il.PagedKV(self.kp, self.vp, self.dev["table"], self.dev["kv_len"], self.dev["cu"])

    def attend(self, **kw):
        return il.ilre_paged_attention(self.dev["q"], self.cache(), max_q=max(self.q_lens), max_kv=max(self.kv_lens), total_kv=sum(self.kv_lens), **kw)

    def check(self, got, lse, absent=None, **kw):
        row = 0
        for s, (a, n) in enumerate(zip(self.q_lens, self.kv_lens)):
            want = oa.attend(_f64(self.q[row:row + a]), _f64(self.k[s]), _f64(self.v[s]), absent=None if absent is None else absent[s], **kw)
            _check(got[row:row + a], lse[row:row + a], *want, n, self.dtype, f"sequence {s}: {a} of {n}")
            row += a


CASES = [
    # q_lens, kv_lens, Hq, Hkv, page, layout, dtype, mask
    ([1], [1], 8, 2, 16, "head", "bf16", {}),
    ([1], [4097], 32, 8, 16, "head", "bf16", {}),
    ([1], [5000], 8, 1, 64, "token", "bf16", {}),
    ([1, 1, 1, 1, 1, 1, 1], [1, 31, 32, 33, 127, 129, 700], 28, 4, 32, "token", "bf16", {}),
    ([1, 0, 1, 3], [5, 0, 900, 3], 8, 2, 16, "head", "bf16", {}),
    ([3, 5], [2, 0], 8, 2, 16, "head", "bf16", {}),                      # rows in front of their sequence see nothing
    ([9], [40], 4, 4, 16, "head", "bf16", {}),
    ([17], [1000], 64, 8, 16, "head", "bf16", {}),                       # 136 rows
    ([8], [777], 28, 4, 64, "head", "bf16", {}),                         # 56 rows
    ([65, 1, 130], [65, 200, 1031], 16, 4, 32, "token", "bf16", {}),
    ([130], [70], 8, 2, 16, "head", "bf16", {}),
    ([100], [3001], 8, 2, 256, "head", "bf16", dict(causal=False)),
    ([1, 2], [300, 2], 8, 2, 16, "head", "bf16", dict(causal=False)),
    ([200, 33], [900, 33], 8, 2, 16, "head", "bf16", dict(sink=4, window=100)),
    ([200], [1500], 8, 2, 64, "head", "bf16", dict(sink=130, window=512)),
    ([70], [400], 4, 4, 16, "token", "bf16", dict(window=1)),
    ([1, 4], [800, 333], 8, 2, 32, "head", "bf16", dict(sink=4, window=64)),
    ([300], [300], 14, 2, 16, "head", "bf16", dict(sink=4, window=37)),
    ([1], [2500], 8, 2, 16, "head", "f32", {}),
    ([1, 7, 0, 50], [33, 7, 4, 333], 8, 2, 32, "token", "f32", {}),
    ([150], [620], 4, 2, 64, "head", "f32", dict(sink=4, window=90)),
    ([40], [500], 28, 4, 16, "head", "f32", dict(causal=False)),
    ([1] * 70, [3 * i + 1 for i in range(70)], 4, 1, 16, "head", "bf16", {}),  # more sequences than a wavefront has lanes
]


@pytest.mark.parametrize("q_lens,kv_lens,Hq,Hkv,page,layout,dtype,mask", CASES,
                         ids=[f"{c[6]}-q{sum(c[0])}-kv{sum(c[1])}-{c[2]}.{c[3]}-p{c[4]}{c[5][0]}-" + ("".join(f"{k}{v}" for k, v in c[7].items()) or "causal") for c in CASES])
def test_paged_attention(q_lens, kv_lens, Hq, Hkv, page, layout, dtype, mask):
    _announce(f"paged {q_lens} of {kv_lens} {Hq}/{Hkv} page {page} {layout} {dtype} {mask}")
    x = Paged(q_lens, kv_lens, Hq, Hkv, page, dtype, layout, seed=sum(kv_lens) + Hq)
    out, lse = x.attend(**mask)
    torch.cuda.synchronize()
    x.check(out, lse, **mask)
    again, lse2 = x.attend(**mask)
    assert torch.equal(out, again) and torch.equal(lse, lse2)
    # a workspace that is not there or too small cuts less, and changes nothing but the rounding
    for ws in (torch.empty(0, dtype=torch.uint8, device="cuda"), torch.empty(sum(q_lens) * Hq * 516 * 2 + 256, dtype=torch.uint8, device="cuda")):
        x.check(*x.attend(workspace=ws, **mask), **mask)


def test_lengths_that_were_promised_otherwise():
    """max_q, max_kv and total_kv only decide how the work is cut up."""
    _announce("paged, promised lengths wrong")
    x = Paged([40, 1, 90], [900, 333, 90], 8, 2, 16, "bf16", seed=3)
    for max_q, max_kv, total in ((1, 1, 1), (1, 16, 5000), (90, 100000, 0), (4000, 900, 100)):
        out, lse = il.ilre_paged_attention(x.dev["q"], x.cache(), max_q=max_q, max_kv=max_kv, total_kv=total)
        x.check(out, lse)


@pytest.mark.parametrize("q_len,mask", [(1, {}), (50, {}), (200, {}), (200, dict(sink=4, window=64)), (1, dict(sink=20, window=64))])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_entries_that_name_no_page(q_len, mask, dtype):
    _announce(f"paged, absent pages, {q_len} new {mask} {dtype}")
    x = Paged([q_len, 3], [1000, 60], 8, 2, 16, dtype, seed=q_len)
    gone = {0: -1, 7: 1 << 30, 20: x.kp.shape[0], 33: -2 ** 31, 61: -5}
    absent = [np.zeros(1000, bool), np.zeros(60, bool)]
    for col, entry in gone.items():
        x.dev["table"][0, col] = entry
        absent[0][col * 16:col * 16 + 16] = True
    out, lse = x.attend(**mask)
    x.check(out, lse, absent=absent, **mask)
    # all of them: the first sequence sees nothing
    x.dev["table"][0] = -1
    out, lse = x.attend(**mask)
    absent[0][:] = True
    x.check(out, lse, absent=absent, **mask)


def test_pages_that_no_row_sees_are_not_looked_at():
    """Streaming: between the sink part and the window the pages may have gone to others, whatever they hold now."""
    _announce("paged, freed pages")
    for q_len in (1, 30, 300):
        x = Paged([q_len], [2000], 8, 2, 16, "bf16", seed=5)
        first = 2000 - q_len - 100 + 1
        for t in range(2000):
            if 4 <= t < first:
                x.kp[x.table[0, t // 16], :, t % 16] = float("nan")
                x.vp[x.table[0, t // 16], :, t % 16] = float("inf")
        freed = [c for c in range(125) if c * 16 >= 16 and c * 16 + 16 <= first]
        out, lse = x.attend(sink=4, window=100)
        x.check(out, lse, sink=4, window=100)
        x.dev["table"][0, freed] = -1
        out2, lse2 = x.attend(sink=4, window=100)
        assert torch.equal(out, out2) and torch.equal(lse, lse2)


def test_boundaries_that_do_not_ascend_stay_within_the_tensors():
    """What comes out then is nobody's business, but it is written inside the outputs and nowhere else, and the call ends."""
    _announce("paged, unordered boundaries")
    x = Paged([40] * 3, [300, 41, 1000], 8, 2, 16, "bf16", seed=21, fill=0.0)
    guard = torch.full((140, 8, 128), 9.0, device="cuda").bfloat16()
    for cu in ([0, 90, 10, 120], [100, 50, 20, 0], [-7, 1 << 30, -(1 << 30), 60], [0, 120, 0, 120]):
        x.dev["cu"].copy_(torch.tensor(cu, dtype=torch.int32))
        for max_q in (1, 40, 120):
            il.ilre_paged_attention(x.dev["q"], x.cache(), max_q=max_q, max_kv=1000, out=guard[10:130])
        il.ilre_rope_append(x.dev["q"], x.dev["q"][:, :2].contiguous(), None, x.cache(), il.ilre_rope_frequencies(128, 1e4), q_out=guard[10:130])
        torch.cuda.synchronize()
        assert (guard[:10] == 9).all() and (guard[130:] == 9).all()


def test_lengths_beyond_the_table_are_cut():
    _announce("paged, kv_len beyond the table")
    x = Paged([3], [64], 8, 2, 16, "bf16", seed=6)
    x.dev["kv_len"].fill_(1 << 30)
    out, lse = x.attend()
    x.check(out, lse)
    x.dev["kv_len"].fill_(-5)
    out, lse = x.attend()
    assert (out == 0).all() and (lse == -float("inf")).all()


@pytest.mark.parametrize("q_len,kv", [(1, 3000), (64, 3000), (300, 3000), (300, 300)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_late_tokens_that_outweigh_everything_before(q_len, kv, dtype):
    """Logits that rise by hundreds of units far behind the first tiles, and ones that fall by as much."""
    _announce(f"paged, rising logits, {q_len} of {kv} {dtype}")
    for sign in (1, -1):
        x = Paged([q_len], [kv], 8, 2, 16, dtype, seed=7)
        step = torch.linspace(-1, 1, kv)[:, None, None] * sign * 40
        u = torch.ones(128)
        x.q = (x.q.float() * 0.1 + u).to(DT[dtype])
        x.k[0] = (x.k[0].float() * 0.1 + step * u).to(DT[dtype])  # logits from -450 to 450
        x.dev["q"] = x.q.cuda()
        kd, t = x.k[0].cuda(), torch.arange(kv)
        x.kp[x.table[0, t // 16].long(), :, (t % 16).cuda()] = kd
        out, lse = x.attend()
        x.check(out, lse)


def test_strides_streams_and_tokens_of_no_sequence():
    _announce("paged, strided q and out, another stream, tokens of no sequence")
    x = Paged([5, 40], [300, 41], 8, 2, 32, "bf16", seed=8)
    T = 45
    wide = torch.randn(T + 6, 12, 128, device="cuda").bfloat16()
    wide[3:3 + T, 2:10] = x.dev["q"]
    outs = torch.full((T + 6, 9, 256), 7.0, device="cuda").bfloat16()
    x.dev["cu"] += 3
    lse = torch.full((T + 6, 8), 7.0, device="cuda")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        out, _ = il.ilre_paged_attention(wide[:, 2:10], x.cache(), max_q=40, max_kv=300, out=outs[:, :8, 128:], lse=lse)
    stream.synchronize()
    assert (outs[:, 8] == 7).all() and (outs[..., :128] == 7).all() and (outs[:3] == 7).all() and (outs[3 + T:] == 7).all()
    assert (lse[:3] == 7).all() and (lse[3 + T:] == 7).all()
    x.check(out[3:3 + T], lse[3:3 + T])


def test_a_captured_step_follows_what_is_written_later():
    _announce("paged, graph")
    x = Paged([1, 1, 1], [700, 33, 2000], 8, 2, 16, "bf16", seed=9)
    cache, q = x.cache(), x.dev["q"]
    ws = il.alloc_workspace_attention(3, 3, 8, 2, 128, 1, 2000)
    out, lse = torch.empty_like(q), torch.empty(3, 8, device="cuda")
    run = lambda: il.ilre_paged_attention(q, cache, max_q=1, max_kv=2000, workspace=ws, out=out, lse=lse)  # noqa: E731
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for lens in ([700, 33, 2000], [1, 30, 1999], [350, 0, 16], [700, 33, 2000]):
        x.dev["kv_len"].copy_(torch.tensor(lens, dtype=torch.int32))
        out.fill_(5.0)
        graph.replay()
        torch.cuda.synchronize()
        got, got_lse = out.clone(), lse.clone()
        run()
        torch.cuda.synchronize()
        assert torch.equal(got, out) and torch.equal(got_lse, lse)
        for s, n in enumerate(lens):
            want = oa.attend(_f64(x.q[s:s + 1]), _f64(x.k[s][:n]), _f64(x.v[s][:n]))
            _check(got[s:s + 1], got_lse[s:s + 1], *want, n, "bf16", f"{lens} {s}")


def test_a_pool_beyond_32_bits():
    """Pages at both ends of a pool of 5 GiB."""
    _announce("paged, pool of 5 GiB")
    pages = 41000
    kp = torch.zeros(pages, 8, 64, 128, dtype=torch.bfloat16, device="cuda")
    vp = torch.zeros_like(kp)
    n, used = 64 * 5, [0, pages - 1, 20000, pages - 2, 32768]
    g = torch.Generator().manual_seed(10)
    k, v, q = (torch.randn(m, h, 128, generator=g).bfloat16() for m, h in ((n, 8), (n, 8), (3, 32)))
    for i, p in enumerate(used):
        kp[p], vp[p] = k[i * 64:i * 64 + 64].transpose(0, 1).cuda(), v[i * 64:i * 64 + 64].transpose(0, 1).cuda()
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    cache = il.PagedKV(kp, vp, i32(used), i32(n), i32(0, 3))
    out, lse = il.ilre_paged_attention(q.cuda(), cache, max_q=3, max_kv=n)
    _check(out, lse, *oa.attend(_f64(q), _f64(k), _f64(v)), n, "bf16")
    # ... and what the append writes there
    f = il.ilre_rope_frequencies(128, 10000.0)
    new = torch.randn(3, 8, 128, generator=g).bfloat16()
    il.ilre_rope_append(None, new.cuda(), new.cuda(), cache, f)
    assert torch.equal(vp[32768, :, 61:].cpu(), new.transpose(0, 1))
    assert torch.equal(vp[32768, :, :61].cpu(), v[256:317].transpose(0, 1))


PROMPTS = [
    ([1], None, 8, 2, "bf16", {}),
    ([33, 1, 129, 300, 0, 64], None, 8, 2, "bf16", {}),
    ([700], None, 28, 4, "bf16", {}),
    ([1200, 5], None, 4, 4, "bf16", {}),
    ([300, 77], [300, 500], 8, 1, "bf16", {}),
    ([300, 77, 9], [300, 0, 5], 8, 2, "bf16", {}),
    ([257, 255], None, 8, 2, "bf16", dict(causal=False)),
    ([600, 100], None, 8, 2, "bf16", dict(sink=4, window=128)),
    ([250, 31], None, 8, 2, "f32", {}),
    ([200, 10], [333, 4], 8, 4, "f32", dict(sink=3, window=50)),
]


@pytest.mark.parametrize("q_lens,k_lens,Hq,Hkv,dtype,mask", PROMPTS, ids=[f"{c[4]}-q{sum(c[0])}-{c[2]}.{c[3]}-{'k' + str(sum(c[1])) if c[1] else 'self'}-{len(c[5])}" for c in PROMPTS])
def test_prompt_attention(q_lens, k_lens, Hq, Hkv, dtype, mask):
    _announce(f"prompt {q_lens} {k_lens} {Hq}/{Hkv} {dtype} {mask}")
    g = torch.Generator().manual_seed(sum(q_lens))
    kl = q_lens if k_lens is None else k_lens
    q = torch.randn(sum(q_lens), Hq, 128, generator=g).to(DT[dtype])
    kv = torch.randn(sum(kl), 2 * Hkv + 1, 128, generator=g).to(DT[dtype])  # keys and values side by side in one row
    k, v = kv[:, :Hkv], kv[:, Hkv + 1:]
    dev = kv.cuda()
    cu = lambda lens: torch.tensor([0] + list(np.cumsum(lens)), dtype=torch.int32, device="cuda")  # noqa: E731
    args = dict(cu_k=None if k_lens is None else cu(k_lens), max_q=max(q_lens), max_k=max(kl), **mask)
    out, lse = il.ilre_prompt_attention(q.cuda(), dev[:, :Hkv], dev[:, Hkv + 1:], cu(q_lens), **args)
    out2, lse2 = il.ilre_prompt_attention(q.cuda(), dev[:, :Hkv], dev[:, Hkv + 1:], cu(q_lens), **args)
    assert torch.equal(out, out2) and torch.equal(lse, lse2)
    row = tok = 0
    for a, n in zip(q_lens, kl):
        want = oa.attend(_f64(q[row:row + a]), _f64(k[tok:tok + n]), _f64(v[tok:tok + n]), **mask)
        _check(out[row:row + a], lse[row:row + a], *want, n, dtype, f"{a} of {n}")
        row, tok = row + a, tok + n


def test_a_neighbour_in_the_packing_may_hold_anything():
    _announce("prompt, NaN in the other sequences")
    T, g = 500, torch.Generator().manual_seed(11)
    q, k, v = (torch.randn(T, h, 128, generator=g).bfloat16() for h in (8, 2, 2))
    for lens, mine in (([100, 333, 67], (100, 433)), ([1, 37, 462], (1, 38))):
        kk, vv = k.clone(), v.clone()
        kk[:mine[0]] = kk[mine[1]:] = float("nan")
        vv[:mine[0]] = vv[mine[1]:] = float("inf")
        cu = torch.tensor([0] + list(np.cumsum(lens)), dtype=torch.int32, device="cuda")
        out, lse = il.ilre_prompt_attention(q.cuda(), kk.cuda(), vv.cuda(), cu, max_q=max(lens))
        s = slice(*mine)
        _check(out[s], lse[s], *oa.attend(_f64(q[s]), _f64(k[s]), _f64(v[s])), mine[1] - mine[0], "bf16")


def test_no_new_tokens_and_no_keys():
    _announce("nothing to do")
    for dtype in DT.values():
        x = Paged([0, 0], [5, 0], 8, 2, 16, "bf16" if dtype == torch.bfloat16 else "f32")
        out, lse = il.ilre_paged_attention(x.dev["q"], x.cache(), max_q=0, max_kv=5)
        assert out.shape == (0, 8, 128) and lse.shape == (0, 8)
        f = il.ilre_rope_frequencies(128, 10000.0)
        e = torch.empty(0, 2, 128, dtype=dtype, device="cuda")
        before = x.kp.clone()
        assert il.ilre_rope(e, f).shape == (0, 2, 128)
        assert il.ilre_rope_append(x.dev["q"], e, e, x.cache(), f).shape == (0, 8, 128)
        assert torch.equal(before.nan_to_num(7.0), x.kp.nan_to_num(7.0))
        cu = torch.zeros(3, dtype=torch.int32, device="cuda")
        out, lse = il.ilre_prompt_attention(x.dev["q"], e, e, cu, max_q=0)
        assert out.shape == (0, 8, 128)
        # queries without a single key
        q = torch.randn(4, 8, 128, device="cuda").to(dtype)
        cu_q = torch.tensor([0, 4], dtype=torch.int32, device="cuda")
        out, lse = il.ilre_prompt_attention(q, e, e, cu_q, cu_k=cu[:2], max_q=4, max_k=0)
        assert (out == 0).all() and (lse == -float("inf")).all()


def test_softmax_scale():
    _announce("prompt, scales")
    g = torch.Generator().manual_seed(12)
    q, k, v = (torch.randn(90, h, 128, generator=g).bfloat16() for h in (4, 2, 2))
    cu = torch.tensor([0, 90], dtype=torch.int32, device="cuda")
    for scale in (0.02, 0.5, 1e-6):
        out, lse = il.ilre_prompt_attention(q.cuda(), k.cuda(), v.cuda(), cu, max_q=90, scale=scale)
        s32 = float(np.float32(scale))
        _check(out, lse, *oa.attend(_f64(q), _f64(k), _f64(v), scale=s32), 90, "bf16")


# ------------------------------------------------------------------------------------------------ rotary positions

def _rope_check(got, x, positions, f, pairing, dtype, rotary):
    """The fraction of a turn reaches fp32 with 2^-25 of half a turn, sines and cosines are off by 2^-23 and rounded with the magnitude, four products and sums
    by 2^-24 each: together less than 2^-21 of the pair's size, before the last rounding."""
    want = oa.rope(_f64(x), positions, np.array(f.inv_freq)[:rotary // 2], f.magnitude, pairing)
    src = np.abs(_f64(x)).max(-1, keepdims=True) * 2 * abs(f.magnitude)
    tol = HALF[dtype] * 1.001 * np.abs(want) + 2.0 ** -21 * src
    assert (np.abs(_f64(got) - want) <= tol).all(), float((np.abs(_f64(got) - want) / tol).max())
    assert torch.equal(got[..., rotary:].cpu(), x[..., rotary:].cpu())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pairing", ["half", "interleaved"])
@pytest.mark.parametrize("rotary", [16, 64, 96, 128])
def test_rope(dtype, pairing, rotary):
    _announce(f"rope {dtype} {pairing} {rotary}")
    code = il.ILRE_ROPE_HALF if pairing == "half" else il.ILRE_ROPE_INTERLEAVED
    f = il.ilre_rope_frequencies(rotary, 500000.0, scaling=il.ILRE_ROPE_PARTS, factor=8.0, low=1.0, high=32.0, original_len=4096)
    g = torch.Generator().manual_seed(rotary)
    for T, H in ((1, 1), (5, 7), (77, 3), (1030, 2)):
        x = torch.randn(T, H, 128, generator=g).to(DT[dtype])
        pos = torch.randint(-2 ** 31, 2 ** 31 - 1, (T,), generator=g).int() if T == 5 else torch.randint(-100, 1100000, (T,), generator=g).int()
        got = il.ilre_rope(x.cuda(), f, pos.cuda(), pairing=code)
        _rope_check(got, x, pos.numpy(), f, pairing, dtype, rotary)
        y = x.cuda()
        assert il.ilre_rope(y, f, pos.cuda(), pairing=code, out=y) is y and torch.equal(y, got)
        got = il.ilre_rope(x.cuda(), f, first_position=999, pairing=code)
        _rope_check(got, x, 999 + np.arange(T), f, pairing, dtype, rotary)


def test_rope_into_the_recalls_key_cache():
    _announce("rope into a key cache")
    f = il.ilre_rope_frequencies(128, 500000.0)
    x = torch.randn(50, 10, 128).bfloat16()
    cache = torch.full((2, 500, 128), 3.0, dtype=torch.bfloat16, device="cuda")
    il.ilre_rope(x.cuda()[:, 3:5], f, first_position=400, out=cache[:, 400:450].transpose(0, 1))
    _rope_check(cache[:, 400:450].transpose(0, 1), x[:, 3:5], 400 + np.arange(50), f, "half", "bf16", 128)
    assert (cache[:, :400] == 3).all() and (cache[:, 450:] == 3).all()


@pytest.mark.parametrize("dtype,layout,pairing", [("bf16", "head", "half"), ("bf16", "token", "interleaved"), ("f32", "head", "interleaved"), ("f32", "token", "half")])
@pytest.mark.parametrize("given", [False, True])
def test_rope_append(dtype, layout, pairing, given):
    _announce(f"append {dtype} {layout} {pairing} positions {given}")
    code = il.ILRE_ROPE_HALF if pairing == "half" else il.ILRE_ROPE_INTERLEAVED
    q_lens, kv_lens = [1, 0, 40, 1100, 3], [700, 5, 40, 1200, 64]
    x = Paged(q_lens, kv_lens, 8, 2, 16, dtype, layout, fill=0.0, seed=13)
    f = il.ilre_rope_frequencies(64, 10000.0)
    T = sum(q_lens)
    g = torch.Generator().manual_seed(14)
    fused = torch.randn(T, 12, 128, generator=g).to(DT[dtype])
    q, k, v = fused[:, :8], fused[:, 8:10], fused[:, 10:]
    places = np.concatenate([np.arange(n - a, n) for a, n in zip(q_lens, kv_lens)])
    positions = places + 12345 if given else places
    k0, v0 = x.kp.clone(), x.vp.clone()
    dev = fused.cuda()
    # the last sequence's new tokens lie on a page that is not there
    x.dev["table"][4, 3] = -1
    got = il.ilre_rope_append(dev[:, :8], dev[:, 8:10], dev[:, 10:], x.cache(), f, torch.tensor(positions, dtype=torch.int32).cuda() if given else None, pairing=code)
    torch.cuda.synchronize()
    _rope_check(got, q, positions, f, pairing, dtype, 64)
    seq = np.repeat(np.arange(5), q_lens)
    stored = seq != 4
    page, cell = x.table[seq, places // 16].long()[torch.tensor(stored)], torch.tensor(places % 16)[torch.tensor(stored)]
    _rope_check(x.kp[page.cuda(), :, cell.cuda()], k[torch.tensor(stored)], positions[stored], f, pairing, dtype, 64)
    assert torch.equal(x.vp[page.cuda(), :, cell.cuda()].cpu(), v[torch.tensor(stored)])
    # nothing else was touched
    k0[page.cuda(), :, cell.cuda()] = x.kp[page.cuda(), :, cell.cuda()]
    v0[page.cuda(), :, cell.cuda()] = x.vp[page.cuda(), :, cell.cuda()]
    assert torch.equal(k0, x.kp) and torch.equal(v0, x.vp)


def test_append_leaves_out_what_has_no_place():
    _announce("append, no place")
    f = il.ilre_rope_frequencies(128, 10000.0)
    for kv in (5, 1000, -3):  # 20 new tokens end at 5: 15 lie in front of the cache; at 1000: behind the table of 4 pages
        kp = torch.zeros(6, 2, 16, 128, device="cuda")
        vp = torch.zeros_like(kp)
        i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
        cache = il.PagedKV(kp, vp, torch.tensor([[4, 2, 0, 1]], dtype=torch.int32, device="cuda"), i32(kv), i32(0, 20))
        x = torch.randn(20, 2, 128, device="cuda")
        q = torch.randn(20, 4, 128, device="cuda")
        got = il.ilre_rope_append(q, x, x, cache, f)
        _rope_check(got, q.cpu(), kv - 20 + np.arange(20), f, "half", "f32", 128)
        if kv == 5:
            assert torch.equal(vp[4, :, :5], x[15:].transpose(0, 1)) and (vp[4, :, 5:] == 0).all()
            vp[4] = 0
        assert (vp == 0).all()
    # keys only
    cache = il.PagedKV(kp, None, torch.tensor([[4, 2, 0, 1]], dtype=torch.int32, device="cuda"), i32(20), i32(0, 20))
    assert il.ilre_rope_append(None, x, None, cache, f) is None
    _rope_check(kp[4].transpose(0, 1), x[:16].cpu(), np.arange(16), f, "half", "f32", 128)


def test_binding_refusals_on_the_device():
    _announce("binding refusals")
    q, k = torch.zeros(2, 8, 128, dtype=torch.bfloat16, device="cuda"), torch.zeros(2, 2, 128, dtype=torch.bfloat16, device="cuda")
    cu = torch.tensor([0, 2], dtype=torch.int32, device="cuda")
    for kw, exc in ((dict(window=-1), il.IlreError), (dict(sink=2), il.IlreError), (dict(causal=False, window=4), il.IlreError),
                    (dict(out=torch.zeros(2, 8, 128, device="cuda")), ValueError), (dict(lse=torch.zeros(2, 4, device="cuda")), ValueError)):
        with pytest.raises(exc):
            il.ilre_prompt_attention(q, k, k, cu, max_q=2, **kw)
    for a, b in ((q[:1].expand(2, 8, 128), k), (q, k[:, :1].expand(2, 2, 128)), (q[:, :1].expand(2, 8, 128), k)):
        with pytest.raises(ValueError):  # a stride of 0 would be taken for contiguous
            il.ilre_prompt_attention(a, b, b, cu, max_q=2)
    i32 = lambda *x: torch.zeros(*x, dtype=torch.int32, device="cuda")  # noqa: E731
    with pytest.raises(ValueError):
        il.PagedKV(torch.zeros(1, 1, 1, 128, device="cuda").expand(4, 2, 16, 128), None, i32(1, 4), i32(1), i32(2))
    with pytest.raises(TypeError):
        il.ilre_prompt_attention(q, k.float(), k.float(), cu, max_q=2)
    with pytest.raises(ValueError):
        il.ilre_prompt_attention(q, k, k, cu.long(), max_q=2)
    with pytest.raises(il.IlreError):
        il.ilre_prompt_attention(q, k.repeat(1, 2, 1)[:, :3].contiguous(), k.repeat(1, 2, 1)[:, :3].contiguous(), cu, max_q=2)
    with pytest.raises(ValueError):
        il.ilre_rope(q, il.ilre_rope_frequencies(128, 1e4), torch.zeros(3, dtype=torch.int32, device="cuda"))


def test_the_example_answers_as_whole_prompts_would():
    """The last token's attention, step by step over the paged cache, against the fp64 attention of everything before it."""
    import importlib.util
    import os

    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "stream_recall_answer.py")
    spec = importlib.util.spec_from_file_location("stream_recall_answer", path)
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    _announce("example")
    r = ex.main(L=3000, budget=300)
    torch.cuda.synchronize()
    assert len(r["idx"]) == 304 and (r["kept"] >= 0).all() and r["answer"].shape == (2, ex.STEPS)
    f = r["freqs"]
    for s, prompt in enumerate(r["prompts"]):
        tokens = torch.cat((prompt.long(), r["answer"][s]))
        q, k, v = r["layer"].project(r["embed"][tokens])
        n = len(tokens)
        q, k = (_f64(il.ilre_rope(t, f)) for t in (q, k))
        # (matrix products over other numbers of tokens may round a state otherwise: its last bit, 2^-8 of it, moves logits by 2^-7 of their reach)
        want, want_lse, size, reach = oa.attend(q[-1:], k, _f64(v))
        got = _f64(r["attended"][s:s + 1])
        tol = HALF["bf16"] * 2 * np.abs(want) + (2 * 2.0 ** -7 * reach[..., None] + 2 * 2.0 ** -8) * size
        assert (np.abs(got - want) <= tol).all(), float((np.abs(got - want) / tol).max())
