"""GPU parity of rotary positions and the fill of a paged cache around and above the number of tokens from which a wavefront has a token to itself."""
import numpy as np
import pytest
import torch

import paper_2508_17892_amd as il
from oracle import attention as oa
from test_gpu_attention import DT, Paged, _announce, _f64, _rope_check

pytestmark = pytest.mark.gpu

CODE = {"half": il.ILRE_ROPE_HALF, "interleaved": il.ILRE_ROPE_INTERLEAVED}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pairing", ["half", "interleaved"])
@pytest.mark.parametrize("rotary", [32, 96, 128])
def test_rope_of_many_tokens(dtype, pairing, rotary):
    _announce(f"rope, many tokens, {dtype} {pairing} {rotary}")
    f = il.ilre_rope_frequencies(rotary, 500000.0, scaling=il.ILRE_ROPE_PARTS, factor=8.0, low=1.0, high=32.0, original_len=4096)
    g = torch.Generator().manual_seed(rotary)
    for T, H in ((4095, 2), (4096, 1), (4099, 37), (9001, 3)):
        x = torch.randn(T, H, 128, generator=g).to(DT[dtype])
        pos = torch.randint(-100, 1100000, (T,), generator=g).int()
        got = il.ilre_rope(x.cuda(), f, pos.cuda(), pairing=CODE[pairing])
        _rope_check(got, x, pos.numpy(), f, pairing, dtype, rotary)
        y = x.cuda()
        assert il.ilre_rope(y, f, pos.cuda(), pairing=CODE[pairing], out=y) is y and torch.equal(y, got)
        got = il.ilre_rope(x.cuda(), f, first_position=999, pairing=CODE[pairing])
        _rope_check(got, x, 999 + np.arange(T), f, pairing, dtype, rotary)


@pytest.mark.parametrize("dtype,layout,pairing", [("bf16", "head", "half"), ("bf16", "token", "interleaved"), ("f32", "head", "interleaved"), ("f32", "token", "half")])
@pytest.mark.parametrize("given", [False, True])
def test_append_of_many_tokens(dtype, layout, pairing, given):
    _announce(f"append, many tokens, {dtype} {layout} {pairing} positions {given}")
    q_lens, kv_lens = [1, 0, 4000, 1100, 3], [700, 5, 4000, 1200, 64]
    x = Paged(q_lens, kv_lens, 8, 2, 16, dtype, layout, fill=0.0, seed=13)
    f = il.ilre_rope_frequencies(64, 10000.0)
    T = sum(q_lens)
    g = torch.Generator().manual_seed(15)
    fused = torch.randn(T + 7, 12, 128, generator=g).to(DT[dtype])  # the last seven tokens are of no sequence
    q, k, v = fused[:, :8], fused[:, 8:10], fused[:, 10:]
    places = np.concatenate([np.arange(n - a, n) for a, n in zip(q_lens, kv_lens)])
    positions = places + 12345 if given else places
    k0, v0 = x.kp.clone(), x.vp.clone()
    dev = fused.cuda()
    # one page of the long sequence and the one of the last sequence's new tokens are not there
    x.dev["table"][2, 100] = x.kp.shape[0]
    x.dev["table"][4, 3] = -1
    out = torch.full((T + 7, 8, 128), 5.0, dtype=DT[dtype], device="cuda")
    pos = torch.tensor(np.append(positions, np.zeros(7)), dtype=torch.int32).cuda() if given else None
    got = il.ilre_rope_append(dev[:, :8], dev[:, 8:10], dev[:, 10:], x.cache(), f, pos, pairing=CODE[pairing], q_out=out)
    torch.cuda.synchronize()
    _rope_check(got[:T], q[:T], positions, f, pairing, dtype, 64)
    assert (got[T:] == 5).all()
    seq = np.repeat(np.arange(5), q_lens)
    stored = torch.tensor((seq != 4) & ~((seq == 2) & (places // 16 == 100)))
    page, cell = x.table[seq, places // 16].long()[stored].cuda(), torch.tensor(places % 16)[stored].cuda()
    _rope_check(x.kp[page, :, cell], k[:T][stored], positions[stored.numpy()], f, pairing, dtype, 64)
    assert torch.equal(x.vp[page, :, cell].cpu(), v[:T][stored])
    # nothing else was touched
    k0[page, :, cell] = x.kp[page, :, cell]
    v0[page, :, cell] = x.vp[page, :, cell]
    assert torch.equal(k0, x.kp) and torch.equal(v0, x.vp)


def test_positions_past_32_bits():
    """first_position + i is the token's position whatever they add up to."""
    _announce("rope, positions around 2^31")
    f = il.ilre_rope_frequencies(128, 500000.0)
    g = torch.Generator().manual_seed(3)
    for T in (9, 4100):
        x = torch.randn(T, 2, 128, generator=g)
        for first in (2 ** 31 - 4, -2 ** 31):
            _rope_check(il.ilre_rope(x.cuda(), f, first_position=first), x, first + np.arange(T), f, "half", "f32", 128)


@pytest.mark.parametrize("pairing", ["half", "interleaved"])
def test_sines_and_cosines_keep_the_bits_of_fp32_where_they_are_small(pairing):
    """One channel of every pair is zero, so that a result is one product, m x cos a or m x sin a, whose error is taken relative to itself.  Angles in fp64 reach
    10^6 positions with less than 2^-33 of a turn lost; sincospi of the fraction's upper part is off by 2 units in the last place (2^-22), what is added for the lower part, the
    magnitude and its rounding, the product and its rounding by 2^-24 each: 9 * 2^-24, with the last rounding 10.  (An angle rounded to fp32 is off by 2^-26 of a
    turn, 1.6 * 2^-24 by itself: more than that share of every cosine below a sixth.)"""
    _announce(f"rope, small sines and cosines, {pairing}")
    for T in (600, 4100):
        f = il.ilre_rope_frequencies(128, 500000.0, scaling=il.ILRE_ROPE_PARTS, factor=8.0, low=1.0, high=32.0, original_len=4096)
        g = torch.Generator().manual_seed(T)
        x = torch.randn(T, 2, 128, generator=g)
        if pairing == "half":
            x[:, 0, :64] = 0
            x[:, 1, 64:] = 0
        else:
            x[:, 0, 0::2] = 0
            x[:, 1, 1::2] = 0
        pos = torch.randint(0, 1000000, (T,), generator=g).int()
        got = _f64(il.ilre_rope(x.cuda(), f, pos.cuda(), pairing=CODE[pairing]))
        want = oa.rope(_f64(x), pos.numpy(), np.array(f.inv_freq), f.magnitude, pairing)
        lost = 2.0 ** -33 * 2 * np.pi * np.abs(_f64(x)).max(-1, keepdims=True) * f.magnitude
        err = np.abs(got - want) / (10 * 2.0 ** -24 * np.abs(want) + lost)
        assert (err <= 1).all(), (float(err.max()), np.argwhere(err > 1)[:3].tolist())
