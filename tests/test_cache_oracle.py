"""Pins of the paged cache's oracle (CPU): each fails for a wrong place, sign, rounding or mask."""
import math

import numpy as np
import pytest
import torch

from oracle import cache_oracle as c
from oracle import taskpress_oracle as o


@pytest.mark.parametrize("d", [64, 128])
def test_places_cover_the_codes_once(d):
    kb, ks, vb, vs = c.places(d)
    nibbles = np.concatenate([(2 * b + s // 4).ravel() for b, s in ((kb, ks), (vb, vs))])
    assert sorted(nibbles) == list(range(2 * 32 * d))
    assert c.block_bytes(d) == {64: 2304, 128: 4480}[d]


def test_places_by_hand():
    # token 1, channel 37 = 32 + 5 of d = 128: s = 1, h = 0, element 5 -> nibble 6: word 16 + 1
    assert c.key_place(128, 1, 37) == (4 * 17 + 3, 0)
    # channel 24 = 8 * 3 of d = 64: h = 3, s = 0, element 0
    assert c.key_place(64, 0, 24) == (4 * 6, 0)
    # token 23 = 16 + 4 + 3: g = 1, element 7 -> nibble 7; channel 70 = 64 + 6: second half, word 256 + 22 * 4
    assert c.value_place(128, 23, 70) == (16 * 128 + 4 * (256 + 88) + 3, 4)
    # channel 35 = 2 * 16 + 3 of token 0
    assert c.value_place(64, 0, 35) == (16 * 64 + 4 * (3 * 4 + 2), 0)


@pytest.mark.parametrize("d", [64, 128])
def test_block_round_trip_leaves_other_tokens(d):
    rng = np.random.default_rng(5)
    block = rng.integers(0, 256, c.block_bytes(d)).astype(np.uint8)
    block[32 * d:] = 0  # finite scales
    before = [x.copy() for x in c.read_block(block, d)]
    k = c.quantise_key(c.to_bf16(rng.normal(size=d)))
    v = c.quantise_value(c.to_bf16(rng.normal(size=d)))
    c.write_token(block, d, 13, k, v)
    kk, vv = c.read_block(block, d)
    assert np.array_equal(kk[13], k[0] * np.repeat(k[1], 32)) and np.array_equal(vv[13], v[0] * np.float64(v[1]))
    others = np.arange(32) != 13
    assert np.array_equal(kk[others], before[0][others]) and np.array_equal(vv[others], before[1][others])


def test_to_bf16():
    rng = np.random.default_rng(6)
    x = np.concatenate([rng.normal(size=5000) * 10.0 ** rng.integers(-38, 38, 5000), [0.0, -0.0, 1.00390625, 1.01171875, 1e-40]])
    x = np.clip(x, -3e38, 3e38).astype(np.float32).astype(np.float64)  # torch rounds from fp32
    assert np.array_equal(c.to_bf16(x), torch.from_numpy(x).float().to(torch.bfloat16).double().numpy())
    assert c.to_bf16(1.00390625 + 2.0 ** -40) == 1.0078125 and c.to_bf16(1.01171875 - 2.0 ** -40) == 1.0078125  # once, not by way of fp32
    assert c.by_fp32(1.00390625 + 2.0 ** -40) == 1.0 and c.by_fp32(1.01171875 - 2.0 ** -40) == 1.015625
    assert c.to_bf16(3.4e38) == c._MAX_BF16 and c.to_bf16(-1e300) == -c._MAX_BF16


def test_key_codes():
    rng = np.random.default_rng(7)
    k = c.to_bf16(rng.normal(size=128) * np.repeat([1.0, 100.0, 1e-3, 0.0], 32))
    codes, scales = c.quantise_key(k)
    assert np.array_equal(scales[:3], c.to_bf16(np.abs(k[:96]).reshape(3, 32).max(1) / 7)) and scales[3] == 0
    assert not codes[96:].any()
    held = codes * np.repeat(scales, 32)
    # half a step, and the scale's rounding (2^-9) times up to 7.5 steps at the largest channel
    assert np.all(np.abs(held - k) <= np.repeat(scales, 32) * (0.5 + 7.5 * 2.0 ** -8))
    assert np.abs(codes[:32]).max() == 7
    # ties go to the even code: scale 1 exactly
    row = np.zeros(64)
    row[:6] = [7.0, 0.5, 1.5, 2.5, -0.5, -3.5]
    assert c.quantise_key(row)[0][:6].tolist() == [7, 0, 2, 2, 0, -4]


def test_value_codes_are_the_quantisers():
    rng = np.random.default_rng(8)
    v = c.to_bf16(rng.standard_t(3, size=(50, 128)))
    g = o.value_scales(v, o.QFMT_INT, 4)
    q = o.quantize_values(v, g, o.QFMT_INT, 4)
    for i in range(50):
        codes, scale = c.quantise_value(v[i])
        assert scale == g[i] and np.array_equal(codes, q[i])


@pytest.mark.parametrize("style", [c.HALVES, c.PAIRS])
def test_rotation(style):
    rng = np.random.default_rng(9)
    x = c.to_bf16(rng.normal(size=64))
    angle = rng.uniform(0, 6, 16)
    cs = np.concatenate([np.cos(angle), np.sin(angle)]).astype(np.float32)
    y = c.rotate(x, cs, 32, style)
    assert np.array_equal(y[32:], x[32:])
    a, b = (x[:16], x[16:32]) if style == c.HALVES else (x[:32:2], x[1:32:2])
    p, q = (y[:16], y[16:32]) if style == c.HALVES else (y[:32:2], y[1:32:2])
    z = (a + 1j * b) * np.exp(1j * angle)  # the pair as a complex number turned by its angle
    assert np.all(np.abs(p + 1j * q - z) <= 2.0 ** -7 * np.abs(z))
    assert np.array_equal(c.rotate(x, np.concatenate([np.ones(16), np.zeros(16)]).astype(np.float32), 32, style), x)


def test_attend():
    rng = np.random.default_rng(10)
    q, k, v = rng.normal(size=8), rng.normal(size=(5, 8)), rng.normal(size=(5, 8))
    seen = np.array([True, False, True, True, False])
    w = [math.exp(0.3 * sum(a * b for a, b in zip(q, k[i]))) if seen[i] else 0.0 for i in range(5)]
    out, lse, _ = c.attend(q, k, v, seen, 0.3)
    assert np.allclose(out, sum(w[i] * v[i] for i in range(5)) / sum(w), atol=1e-14)
    assert abs(lse - math.log(sum(w))) < 1e-14
    out, lse, _ = c.attend(q, k, v, np.zeros(5, dtype=bool), 0.3)
    assert not out.any() and lse == -math.inf


def test_missing_page():
    assert c.place_of([4, -1, 9], 9, 64, 70) is None and c.place_of([4, -1, 9], 9, 64, 128) is None
    assert c.place_of([4, -1, 8], 9, 64, 63) == (4, 1, 31) and c.place_of([4, -1, 8], 9, 64, 128 + 33) == (8, 1, 1)
