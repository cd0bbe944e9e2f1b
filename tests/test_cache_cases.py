"""The bounds of cache_cases.py refuse wrong outputs on every input that the GPU tests use them on."""
import math

import numpy as np
import pytest

import cache_cases as cc
import test_gpu_cache as T


class Host(T.Setup):
    def upload(self):
        pass


@pytest.mark.parametrize("shape", range(len(cc.SHAPES)))
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kind", cc.KINDS)
def test_wrong_outputs_are_refused(kind, d, shape):
    Hq, Hkv, lens, new, _ = cc.SHAPES[shape]
    s = Host(80 + shape, 1, Hq, Hkv, d, 64, lens)
    q, scale = cc.fill(s, kind, sum(new))
    for row, hq, bound in cc.rows(s, new, q, scale):
        ref, lse = bound[0], bound[1]
        assert cc.accepts(ref, lse, bound)
        if lse == -math.inf:
            continue
        for wrong in (0 * ref, -ref, 1.1 * ref, 0.9 * ref, 3 * ref, ref + 0.1 * np.abs(ref).max()):
            assert not cc.accepts(wrong, lse, bound), (row, hq)
        for off in (0.1, -0.1, math.log(2), -1000.0):
            assert not cc.accepts(ref, lse + off, bound), (row, hq)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kind", ["weak", "levels", "massive"])
def test_lost_scales_are_refused(kind, d):
    """Key scales 2^19 below the largest of their block taken as 0: refused in most rows of the kinds made for it."""
    from oracle import cache_oracle as c

    Hq, Hkv, lens, new, _ = cc.SHAPES[0]
    s = Host(80, 1, Hq, Hkv, d, 64, lens)
    q, scale = cc.fill(s, kind, sum(new))
    right = list(cc.rows(s, new, q, scale))
    blocks = s.pages.reshape(-1, c.block_bytes(d))
    ks = (blocks[:, 32 * d:34 * d].copy().view(np.uint16).astype(np.uint32) << 16).view(np.float32)
    ks[ks < ks.max(1, keepdims=True) * 2.0 ** -19] = 0
    blocks[:, 32 * d:34 * d] = c.bf16_bits(ks).view(np.uint8).reshape(len(blocks), -1)
    lost = list(cc.rows(s, new, q, scale))
    refused = [not cc.accepts(b[0], b[1], a) for (_, _, a), (_, _, b) in zip(right, lost)]
    assert np.mean(refused) > 0.9
