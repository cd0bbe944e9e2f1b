"""Pins of the 8-bit cache's oracle (CPU): each fails for a wrong place, rounding or scale."""
import numpy as np
import pytest

from oracle import cache8_oracle as c
from oracle import cache_oracle as c4
from oracle import taskpress_oracle as o


@pytest.mark.parametrize("d", [64, 128])
def test_places_cover_the_codes_once(d):
    k, v = c.places(d)
    assert sorted(np.concatenate([k.ravel(), v.ravel()])) == list(range(64 * d))
    assert c.block_bytes(d) == {64: 4240, 128: 8336}[d]


def test_places_by_hand():
    # token 17 = tile 1, row 1; channel 101 = 64 + 32 + 5: second kilobyte, product 3 (its pair's second), channels 0..7
    assert c.key_place(128, 17, 101) == 2048 + 1024 + 1 * 16 + 8 + 5
    # channel 30 = 3 * 8 + 6 of d = 64: lanes 48.., the pair's first
    assert c.key_place(64, 2, 30) == (48 + 2) * 16 + 6
    # token 23 = 16 + 4 + 3: lanes 16.., byte 7; channel 70 = 2 * 32 + 6: tile 4, the first of its pair
    assert c.value_place(128, 23, 70) == 32 * 128 + 2048 + (16 + 6) * 16 + 7
    # channel 20 = 16 + 4 of token 2: the pair's second
    assert c.value_place(64, 2, 20) == 32 * 64 + 4 * 16 + 8 + 2


@pytest.mark.parametrize("fmt", [c.INT, c.FP8])
@pytest.mark.parametrize("d", [64, 128])
def test_block_round_trip_leaves_other_tokens(d, fmt):
    rng = np.random.default_rng(5)
    block = c.bytes_of(rng.normal(size=c.block_bytes(d)) * 30, fmt)
    block[64 * d:] = np.full(36, 0.25, dtype=np.float32).view(np.uint8)
    before = [x.copy() for x in c.read_block(block, d, fmt)]
    k, v = (c4.to_bf16(rng.normal(size=d)) for _ in range(2))
    c.write_keys(block, d, fmt, 13, {13: k})
    c.write_value(block, d, 13, *c.quantise_value(v, fmt))
    kk, vv = c.read_block(block, d, fmt)
    g = np.abs(v).max() / c.qmax(fmt)
    for got, want, step in ((kk[13], k, 0.25), (vv[13], v, g)):  # e4m3: half of 2^-3 of the number, or of 2^-9 steps
        most = step * 0.51 if fmt == c.INT else np.maximum(np.abs(want) * 2.0 ** -4 * 1.01, step * 2.0 ** -10 * 1.01)
        assert np.all(np.abs(got - want) <= most)
    others = np.arange(32) != 13
    assert np.array_equal(kk[others], before[0][others]) and np.array_equal(vv[others], before[1][others])


def test_bytes():
    assert c.bytes_of([0.5, 1.5, -2.5, 126.5, 200, -200], c.INT).tolist() == [128, 130, 126, 254, 255, 1]
    assert c.codes_of(np.array([1, 128, 255], dtype=np.uint8), c.INT).tolist() == [-127, 0, 127]
    assert c.bytes_of([448, 460, -0.0, 2.0 ** -9, 2.0 ** -10, 17.0], c.FP8).tolist() == [0x7E, 0x7E, 0x80, 1, 0, 0x58]
    assert c.codes_of(np.array([0x7E, 0x81, 0x38], dtype=np.uint8), c.FP8).tolist() == [448, -2.0 ** -9, 1.0]


@pytest.mark.parametrize("fmt", [c.INT, c.FP8])
def test_scale_of_a_fresh_block_and_its_rise(fmt):
    d, rng = 64, np.random.default_rng(6)
    Q = c.qmax(fmt)
    block = rng.integers(0, 255, c.block_bytes(d)).astype(np.uint8)  # whatever
    keys = {t: c4.to_bf16(rng.normal(size=d)) for t in (0, 1, 2)}
    c.write_keys(block, d, fmt, 0, keys)
    m = max(np.abs(k).max() for k in keys.values())
    first = c.key_scale(block, d)
    assert first == np.float32(m / Q)
    was = c.read_block(block, d, fmt)[0][:3]
    c.write_keys(block, d, fmt, 3, {3: np.full(d, m)})  # as large as the scale holds
    assert c.key_scale(block, d) == first and np.array_equal(c.read_block(block, d, fmt)[0][:3], was)
    more = np.zeros(d)
    more[5] = float(c4.to_bf16(m * 1.01))
    c.write_keys(block, d, fmt, 4, {4: more})
    assert c.key_scale(block, d) == 2 * first
    more[5] *= 9
    c.write_keys(block, d, fmt, 5, {5: more})
    assert c.key_scale(block, d) == 16 * first
    got = c.read_block(block, d, fmt)[0]
    for t, k in keys.items():
        off = np.abs(got[t] - k)
        if fmt == c.INT:  # 1/2 (1 + 1/8 + 1/16) of a step
            assert np.all(off <= 16 * first * 0.6)
        else:  # 2^-4, or half a subnormal step of each scale
            assert np.all(off <= np.maximum(np.abs(k) * 2.0 ** -4 * 1.01, first * 16 * 2.0 ** -9))
    assert abs(got[5, 5] - more[5]) <= 16 * first * (0.5 if fmt == c.INT else 16)


def test_no_scale_and_strange_scales():
    d = 64
    for held in (0.0, -1.0, np.nan):
        block = np.full(c.block_bytes(d), 200, dtype=np.uint8)
        block[64 * d + 128:64 * d + 132] = np.array([held], dtype=np.float32).view(np.uint8)
        c.write_keys(block, d, c.INT, 2, {2: np.full(d, 1.27)})
        assert c.key_scale(block, d) == np.float32(1.27 / 127)
        assert np.all(block[c.places(d)[0][0]] == 200)  # what is before keeps its codes
    block = np.full(c.block_bytes(d), 200, dtype=np.uint8)
    c.write_keys(block, d, c.INT, 0, {0: np.zeros(d)})
    assert c.key_scale(block, d) == 0 and np.all(block[c.places(d)[0][0]] == 128)


@pytest.mark.parametrize("fmt", [c.INT, c.FP8])
@pytest.mark.parametrize("held", [np.inf, -np.inf])
def test_an_infinite_scale_is_none(held, fmt):
    d = 64
    block = np.full(c.block_bytes(d), 0x48, dtype=np.uint8)
    block[64 * d + 128:64 * d + 132] = np.array([held], dtype=np.float32).view(np.uint8)
    c.write_keys(block, d, fmt, 2, {2: np.full(d, 1.25)})
    assert c.key_scale(block, d) == np.float32(1.25 / c.qmax(fmt))
    assert np.all(block[c.places(d)[0][0]] == 0x48) and np.all(c.codes_of(block[c.places(d)[0][2]], fmt) == c.qmax(fmt))


@pytest.mark.parametrize("fmt", [c.INT, c.FP8])
def test_values_are_the_quantisers(fmt):
    rng = np.random.default_rng(8)
    v = c4.to_bf16(rng.standard_t(3, size=(50, 128)))
    g = o.value_scales(v, fmt, 8)
    q = o.pack_codes(o.quantize_values(v, g, fmt, 8), fmt, 8)
    for i in range(50):
        got, scale = c.quantise_value(v[i], fmt)
        assert scale == g[i] and np.array_equal(got ^ (0 if fmt == c.FP8 else 128), q[i])
