"""The attention's plan on the host: chunks cover the length bound, and the partial results of any call fit the
workspace that the plan asks for."""
import ctypes

import numpy as np

from paper_2608_03276_amd import binding as B


class Plan(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("tiles", "row_groups", "chunk", "chunks", "waves", "once")] + \
               [(n, ctypes.c_size_t) for n in ("stat_off", "o_off", "total")]


plan_of = B.load()._ZN2tp10cache_planEiiiiiii  # tp::cache_plan(L, Hq, Hkv, head_dim, batch, max_new, max_len)
plan_of.restype = Plan
plan_of.argtypes = [ctypes.c_int32] * 7


def check(L, R, Hkv, d, batch, most, length):
    p = plan_of(L, R * Hkv, Hkv, d, batch, most, length)
    rows, heads = R * most, L * Hkv * batch
    case = (L, R, Hkv, d, batch, most, length)
    assert p.tiles in (1, 2, 4) and p.tiles * p.row_groups * 16 >= rows > (p.row_groups - 1) * p.tiles * 16, case
    assert p.chunk % 128 == 0 and p.chunk * p.chunks >= length > p.chunk * (p.chunks - 1), case
    assert p.waves in (4, 8) and (p.waves == 4 or (p.tiles == 1 and p.chunks == 1)), case
    partial = heads * rows * p.chunks if p.chunks > 1 else 0
    assert p.stat_off == 0 and p.o_off % 256 == 0 and partial * 8 <= p.o_off and p.o_off + partial * d * 4 <= p.total, case
    return p


def test_partial_results_fit_the_workspace():
    rng = np.random.default_rng(4)
    seen = set()
    for _ in range(60000):
        L, Hkv, R = (int(rng.choice(x)) for x in ([1, 1, 2, 32], [1, 2, 5, 8], [1, 2, 4, 5, 8, 16, 64]))
        batch, most, length = (int(np.exp(rng.uniform(0, np.log(x)))) for x in (2000, 4000, 1 << 30))
        p = check(L, R, Hkv, int(rng.choice([64, 128])), batch, most, length)
        seen.add((p.tiles, p.chunks > 1, p.waves))
    assert seen == {(1, False, 4), (1, False, 8), (1, True, 4), (2, False, 4), (2, True, 4), (4, False, 4), (4, True, 4)}


def test_streaming_with_eight_waves_is_for_large_heads_only():
    """The one combination of eight waves and d = 64 that no kernel exists for."""
    for heads in range(1, 600):
        for length in (4096, 4095, 4097, 2048, 1 << 20):
            p = check(1, 1, 1, 64, heads, 1, length)
            assert p.waves == 4 or not p.once
    assert check(1, 1, 1, 128, 512, 1, 4096).waves == 8 and check(1, 1, 1, 128, 512, 1, 4096).once
