"""The 8-bit cache's plan on the host: chunks cover the length bound, and the partial results of any call, in chunks or in
shares, fit the workspace that the plan asks for."""
import ctypes

import numpy as np

from paper_2608_03276_amd import binding as B
from test_cache_plan import Plan

plan_of = B.load()._ZN2tp11cache8_planEiiiiiii  # tp::cache8_plan(L, Hq, Hkv, head_dim, batch, max_new, max_len)
plan_of.restype = Plan
plan_of.argtypes = [ctypes.c_int32] * 7
LEAST, START = 4, 4  # blocks of a share at least, and what a pair's start counts


def check(L, R, Hkv, d, batch, most, length):
    p = plan_of(L, R * Hkv, Hkv, d, batch, most, length)
    rows, heads = R * most, L * Hkv * batch
    case = (L, R, Hkv, d, batch, most, length)
    assert p.tiles in (1, 2, 4) and p.tiles * p.row_groups * 16 >= rows > (p.row_groups - 1) * p.tiles * 16, case
    assert p.o_off % 256 == 0 and p.stat_off == 0, case
    if p.chunk == 0:  # shares
        assert p.tiles < 4 and p.row_groups == 1 and batch <= 1024 and p.chunks > 1, case
        every = heads * ((length + 31) // 32 + START)  # of all pairs
        assert every < 1 << 31, case
        used = min(p.chunks, -(-every // LEAST))
        partial = used * 2 * 16 * p.tiles
    else:
        assert p.chunk % 128 == 0 and p.chunk * p.chunks >= length > p.chunk * (p.chunks - 1), case
        assert p.waves in (4, 8) and (p.waves == 4 or (p.tiles == 1 and p.chunks == 1)), case
        partial = heads * rows * p.chunks if p.chunks > 1 else 0
    assert partial * 8 <= p.o_off and p.o_off + partial * d * 4 <= p.total, case
    return p


def test_partial_results_fit_the_workspace():
    rng = np.random.default_rng(4)
    seen = set()
    for _ in range(60000):
        L, Hkv, R = (int(rng.choice(x)) for x in ([1, 1, 2, 32], [1, 2, 5, 8], [1, 2, 4, 5, 8, 16, 64]))
        batch, most, length = (int(np.exp(rng.uniform(0, np.log(x)))) for x in (5000, 4000, 1 << 30))
        p = check(L, R, Hkv, int(rng.choice([64, 128])), batch, most, length)
        seen.add((p.tiles, p.chunks > 1, p.chunk == 0, p.waves if p.chunk else 0))
    assert seen >= {(1, False, False, 4), (1, False, False, 8), (1, True, True, 0), (1, True, False, 4), (2, False, False, 4),
                    (2, True, True, 0), (2, True, False, 4), (4, False, False, 4), (4, True, False, 4)}


def test_what_is_not_split_is_as_in_the_4_bit_cache():
    four = B.load()._ZN2tp10cache_planEiiiiiii
    four.restype, four.argtypes = Plan, [ctypes.c_int32] * 7
    rng = np.random.default_rng(5)
    for _ in range(5000):
        args = (1, 8 * int(rng.choice([1, 4, 8])), 8, int(rng.choice([64, 128])), int(rng.integers(1, 200)), int(rng.integers(1, 40)),
                int(np.exp(rng.uniform(0, 12))))
        a, b = plan_of(*args), four(*args)
        assert (a.tiles, a.row_groups) == (b.tiles, b.row_groups)
        if a.chunk:
            assert (a.chunk, a.chunks, a.waves) == (b.chunk, b.chunks, b.waves)
        else:
            assert b.chunks > 1 and b.tiles < 4
