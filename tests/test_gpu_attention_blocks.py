"""GPU parity of the attention kernels where a call is cut into blocks and ranges, against the fp64 oracle; tolerances as in test_gpu_attention."""
import numpy as np
import pytest
import torch

import paper_2508_17892_amd as il
from oracle import attention as oa
from test_gpu_attention import DT, Paged, _announce, _check, _f64

pytestmark = pytest.mark.gpu


class Packed:
    """Random packed prompts, keys and values side by side in one row."""

    def __init__(self, lens, Hq, Hkv, dtype, seed):
        g = torch.Generator().manual_seed(seed)
        self.lens, self.dtype, self.Hq, self.Hkv = lens, dtype, Hq, Hkv
        self.q = torch.randn(sum(lens), Hq, 128, generator=g).to(DT[dtype])
        self.kv = torch.randn(sum(lens), 2 * Hkv + 1, 128, generator=g).to(DT[dtype])
        self.dev = self.q.cuda(), self.kv.cuda(), torch.tensor([0] + list(np.cumsum(lens)), dtype=torch.int32, device="cuda")

    def attend(self, **kw):
        q, kv, cu = self.dev
        return il.ilre_prompt_attention(q, kv[:, :self.Hkv], kv[:, self.Hkv + 1:], cu, max_q=max(self.lens), **kw)

    def workspace(self):
        return il.alloc_workspace_attention(sum(self.lens), len(self.lens), self.Hq, self.Hkv, 128, max(self.lens), max(self.lens), total_kv=sum(self.lens),
                                            dtype=il.ILRE_BF16 if self.dtype == "bf16" else il.ILRE_F32)

    def check(self, out, lse, **mask):
        row = 0
        for n in self.lens:
            s = slice(row, row + n)
            _check(out[s], lse[s], *oa.attend(_f64(self.q[s]), _f64(self.kv[s, :self.Hkv]), _f64(self.kv[s, self.Hkv + 1:]), **mask), n, self.dtype, f"{n} tokens")
            row += n


def _workspace_of(x, Hq, Hkv):
    return il.alloc_workspace_attention(sum(x.q_lens), len(x.q_lens), Hq, Hkv, 128, max(x.q_lens), max(x.kv_lens), total_kv=sum(x.kv_lens),
                                        dtype=il.ILRE_BF16 if x.dtype == "bf16" else il.ILRE_F32)


# The last block of a sequence, often of a single row, sees fewer tiles of its window than a full one, and lists are cut into ranges right in between.
STREAMS = [
    # q_lens, kv_lens, Hq, Hkv, dtype, sink, window
    ([14, 132], [295, 528], 1, 1, "bf16", 4, 320),
    ([129, 129], [600, 600], 4, 4, "bf16", 4, 320),
    ([388, 79], [2725, 2332], 4, 4, "bf16", 4, 64),
    ([262, 27, 16], [1623, 363, 332], 1, 1, "bf16", 140, 1173),
    ([97, 282, 254], [1166, 1820, 576], 16, 8, "bf16", 168, 1183),
    ([215, 69, 79], [1216, 382, 612], 3, 1, "bf16", 4, 624),
    ([158, 63, 6], [1273, 638, 1074], 20, 4, "bf16", 4, 622),
    ([134, 0], [364, 109], 1, 1, "f32", 4, 192),
    ([150, 150], [900, 900], 8, 8, "f32", 4, 512),
    ([46, 76], [18, 303], 4, 2, "f32", 4, 97),
    ([392, 444], [2019, 1118], 12, 4, "f32", 4, 512),
    ([139, 129], [509, 286], 5, 1, "f32", 20, 240),
    ([249, 148], [255, 464], 7, 1, "f32", 4, 113),
]


@pytest.mark.parametrize("q_lens,kv_lens,Hq,Hkv,dtype,sink,window", STREAMS, ids=[f"{c[4]}-{c[2]}.{c[3]}-q{sum(c[0])}-kv{sum(c[1])}-w{c[6]}" for c in STREAMS])
def test_streamed_chunks_of_several_sequences(q_lens, kv_lens, Hq, Hkv, dtype, sink, window):
    _announce(f"streams {q_lens} of {kv_lens} {Hq}/{Hkv} {dtype} sink {sink} window {window}")
    x = Paged(q_lens, kv_lens, Hq, Hkv, 16, dtype, seed=sum(kv_lens) + Hq)
    ws = _workspace_of(x, Hq, Hkv)
    ws.fill_(255)  # NaN, in the partial results and their logarithms: what no workgroup writes must not be added up
    out, lse = x.attend(sink=sink, window=window, workspace=ws)
    torch.cuda.synchronize()
    x.check(out, lse, sink=sink, window=window)


PACKED = [
    ([171, 0, 285], 1, 1, "f32", 4, 70),
    ([104, 223], 3, 1, "f32", 4, 39),
    ([282, 229], 20, 4, "f32", 4, 58),
    ([15, 221], 7, 1, "f32", 4, 59),
    ([700, 300, 513], 4, 4, "bf16", 4, 128),
]


@pytest.mark.parametrize("lens,Hq,Hkv,dtype,sink,window", PACKED, ids=[f"{c[3]}-{c[1]}.{c[2]}-{sum(c[0])}-w{c[5]}" for c in PACKED])
def test_packed_prompts_with_a_window(lens, Hq, Hkv, dtype, sink, window):
    _announce(f"packed {lens} {Hq}/{Hkv} {dtype} sink {sink} window {window}")
    x = Packed(lens, Hq, Hkv, dtype, sum(lens))
    ws = x.workspace()
    ws.fill_(255)
    out, lse = x.attend(sink=sink, window=window, workspace=ws)
    torch.cuda.synchronize()
    x.check(out, lse, sink=sink, window=window)


def test_a_stream_that_lies_evenly_over_the_tiles_takes_no_longer():
    """Where the window begins with a tile, a wavefront whose half of the sink tile holds nothing has seen nothing before the first whole tile: its rows take their
    references from there.  (Weights against no reference send the workgroup through its tiles a second time, 1.6 times as long.)"""
    _announce("stream, 9216 and 9220 tokens")
    calls = []
    for kv in (9216, 9220):
        x = Paged([1024], [kv], 16, 4, 64, "bf16", seed=kv)
        cache, ws = x.cache(), _workspace_of(x, 16, 4)
        out, lse = x.attend(sink=4, window=512)
        rows = torch.tensor(sorted({0, 1, 31, 32, 63, 64, 65, 500, 991, 992, 1023}))
        for i in rows.tolist():  # a row alone, at the end of what it may see
            n = kv - 1024 + i + 1
            want = oa.attend(_f64(x.q[i:i + 1]), _f64(x.k[0][:n]), _f64(x.v[0][:n]), sink=4, window=512)
            _check(out[i:i + 1], lse[i:i + 1], *want, 516, "bf16", f"row {i} of {kv}")
        calls.append(lambda x=x, cache=cache, ws=ws, out=out, lse=lse: il.ilre_paged_attention(x.dev["q"], cache, max_q=1024, max_kv=max(x.kv_lens), sink=4, window=512,
                                                                                             workspace=ws, out=out, lse=lse))
    begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    best = [float("inf"), float("inf")]
    for _ in range(15):
        for i, call in enumerate(calls):
            call()
            begin.record()
            for _ in range(40):
                call()
            end.record()
            end.synchronize()
            best[i] = min(best[i], begin.elapsed_time(end))
    assert best[0] < 1.25 * best[1], best


# Calls whose blocks have 256 rows: lists of more than 24 tiles, or blocks enough for every compute unit; and the other kernels where they are cut into ranges.
PROMPTS = [
    # q_lens, Hq, Hkv, dtype, mask
    ([1700], 2, 1, "bf16", {}),
    ([1600, 5, 1801, 257], 4, 2, "bf16", {}),
    ([1601, 300], 7, 1, "bf16", {}),
    ([1921], 3, 3, "bf16", {}),
    ([1600, 1], 8, 1, "bf16", dict(causal=False)),
    ([2300, 333], 4, 4, "bf16", dict(sink=4, window=1500)),
    ([1800, 1], 4, 1, "bf16", dict(sink=70, window=1472)),
    ([1024, 33], 64, 8, "bf16", dict(sink=4, window=100)),
    ([1100], 5, 1, "f32", {}),
    ([9], 5, 1, "f32", {}),
    ([9, 1, 20], 3, 1, "bf16", {}),
    ([5, 1, 8], 4, 1, "f32", {}),
]


@pytest.mark.parametrize("lens,Hq,Hkv,dtype,mask", PROMPTS, ids=[f"{c[3]}-{c[1]}.{c[2]}-{sum(c[0])}-" + ("".join(f"{k}{v}" for k, v in c[4].items()) or "causal") for c in PROMPTS])
def test_prompts_in_every_kind_of_block(lens, Hq, Hkv, dtype, mask):
    _announce(f"prompts {lens} {Hq}/{Hkv} {dtype} {mask}")
    x = Packed(lens, Hq, Hkv, dtype, sum(lens) + Hq)
    ws = x.workspace()
    ws.fill_(255)
    out, lse = x.attend(workspace=ws, **mask)
    torch.cuda.synchronize()
    x.check(out, lse, **mask)
    again, lse2 = x.attend(workspace=ws, **mask)
    assert torch.equal(out, again) and torch.equal(lse, lse2)


def test_long_prompts_beside_neighbours_that_may_hold_anything():
    _announce("prompts of 1700 tokens, NaN in the other sequences")
    for lens, mine in (([100, 1700, 67], (100, 1800)), ([1700, 1650], (1700, 3350))):
        x = Packed(lens, 4, 1, "bf16", sum(lens))
        q, kv, cu = x.dev
        for a, b in ((0, mine[0]), (mine[1], sum(lens))):
            kv[a:b, :1] = float("nan")
            kv[a:b, 2:] = float("inf")
        out, lse = x.attend()
        s = slice(*mine)
        _check(out[s], lse[s], *oa.attend(_f64(x.q[s]), _f64(x.kv[s, :1]), _f64(x.kv[s, 2:])), mine[1] - mine[0], "bf16")


@pytest.mark.parametrize("lens", [[1700, 129], [700]])
def test_prompts_whose_late_tokens_outweigh_everything_before(lens):
    """Logits that rise, or fall, by hundreds of units along a prompt."""
    _announce(f"prompts, rising logits, {lens}")
    for sign in (1, -1):
        x = Packed(lens, 4, 2, "bf16", 7)
        step = torch.cat([torch.linspace(-1, 1, n) for n in lens])[:, None, None] * sign * 40
        x.q = (x.q.float() * 0.1 + 1).bfloat16()
        x.kv[:, :2] = (x.kv[:, :2].float() * 0.1 + step).bfloat16()
        x.dev = x.q.cuda(), x.kv.cuda(), x.dev[2]
        x.check(*x.attend())


# The same over pages.
CHUNKS = [
    # q_lens, kv_lens, Hq, Hkv, page, layout, dtype, mask
    ([300], [2000], 2, 1, 16, "head", "bf16", {}),
    ([257, 90, 1], [1700, 2100, 5], 8, 2, 32, "token", "bf16", {}),
    ([150], [1601], 14, 2, 64, "head", "bf16", {}),
    ([200, 64], [1800, 64], 8, 1, 16, "head", "bf16", dict(causal=False)),
    ([400, 131], [2600, 1900], 4, 4, 16, "head", "bf16", dict(sink=4, window=1600)),
    ([600], [2304], 4, 1, 64, "token", "bf16", dict(sink=4, window=1472)),
    ([1024, 40], [1500, 700], 64, 8, 64, "head", "bf16", dict(sink=4, window=100)),
    ([1, 1], [2000, 9], 4, 1, 16, "head", "f32", {}),
    ([60], [700], 5, 1, 16, "token", "f32", {}),
    ([9], [40], 5, 1, 16, "head", "f32", {}),
]


@pytest.mark.parametrize("q_lens,kv_lens,Hq,Hkv,page,layout,dtype,mask", CHUNKS,
                         ids=[f"{c[6]}-q{sum(c[0])}-kv{sum(c[1])}-{c[2]}.{c[3]}-" + ("".join(f"{k}{v}" for k, v in c[7].items()) or "causal") for c in CHUNKS])
def test_chunks_in_every_kind_of_block(q_lens, kv_lens, Hq, Hkv, page, layout, dtype, mask):
    _announce(f"chunks {q_lens} of {kv_lens} {Hq}/{Hkv} page {page} {layout} {dtype} {mask}")
    x = Paged(q_lens, kv_lens, Hq, Hkv, page, dtype, layout, seed=sum(kv_lens) + Hq)
    ws = _workspace_of(x, Hq, Hkv)
    ws.fill_(255)
    out, lse = x.attend(workspace=ws, **mask)
    torch.cuda.synchronize()
    x.check(out, lse, **mask)
    # pages that are not there: the first one, some in between, the last one
    absent = []
    for s, n in enumerate(kv_lens):
        gone = np.zeros(n, bool)
        for col in {0, 3, n // page // 2, (n - 1) // page}:
            x.dev["table"][s, min(col, x.table.shape[1] - 1)] = (-1, 1 << 30, x.kp.shape[0])[col % 3]
            gone[col * page:col * page + page] = True
        absent.append(gone)
    out, lse = x.attend(workspace=ws, **mask)
    x.check(out, lse, absent=absent, **mask)
