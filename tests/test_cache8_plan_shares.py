"""The division of a decoding call into shares, as the kernels form it on the device, against the plan that the host
makes for it: what any lengths write fits the workspace, and every position is below 2^31.  The constants are the source's."""
import os
import re

import numpy as np
import pytest

import test_cache8_plan as P

SOURCE = os.path.join(os.path.dirname(P.B.__file__), "csrc", "cache8_attention.hip")


def constant(name):
    with open(SOURCE) as f:
        return int(re.search(rf"constexpr int {name} = (\d+);", f.read()).group(1))


START, LEAST, MOST = (constant(n) for n in ("kStart", "kLeastShare", "kMostSequences"))


def division(lens, heads, workgroups, start=START):
    """All positions, those of a share, and the workgroups that have any (share_of, k_cache8_shares)."""
    every = sum(max(-(-n // 32), 1) + start for n in lens) * heads
    share = max((-(-every // workgroups) + 3) // 4 * 4, LEAST)
    return every, share, -(-every // share)


def parts(lens, heads, workgroups):
    """The slots of partial results that are written and those that are joined, as (sequence, head) -> [slot]."""
    every, share, used = division(lens, heads, workgroups)
    written, joined, at = {}, {}, 0
    for b, n in enumerate(lens):
        blocks = max(-(-n // 32), 1)
        length = blocks + START
        for lh in range(heads):
            w0, w1 = (at + START) // share, (at + length - 1) // share
            if w0 != w1:
                joined[b, lh] = [2 * w + (w == w0) for w in range(w0, w1 + 1)]
            taken = 0
            for w in range(at // share, w1 + 1):  # the workgroup's part of the pair
                lo, hi = max(at, w * share) - at, min(at + length, (w + 1) * share) - at
                first, stop = max(lo - START, 0), hi - START
                if stop <= first:
                    continue
                assert first == taken
                taken = stop
                if not (first == 0 and stop == blocks):
                    written.setdefault((b, lh), []).append(2 * w + (first == 0))
            assert taken == blocks
            at += length
    assert at == every
    return written, joined, used


def test_parts_are_written_once_and_all_of_them_joined():
    rng = np.random.default_rng(6)
    for _ in range(300):
        lens = [int(np.exp(rng.uniform(0, np.log(rng.choice([40, 3000, 60000]))))) - 1 for _ in range(int(rng.integers(1, 40)))]
        written, joined, used = parts(lens, int(rng.choice([1, 2, 8, 24])), 256)
        assert written == joined and used <= 256
        slots = [s for x in written.values() for s in x]
        assert len(set(slots)) == len(slots) and all(s < 2 * used for s in slots)


def slots_that_fit(p, d):
    return min(p.o_off // 8, (p.total - p.o_off) // (4 * d)) // (16 * p.tiles)


def cases():
    rng = np.random.default_rng(7)
    for _ in range(20000):
        L, Hkv, R = (int(rng.choice(x)) for x in ([1, 1, 2, 32], [1, 2, 5, 8], [1, 2, 4, 5, 8, 16]))
        batch = int(np.exp(rng.uniform(0, np.log(MOST + 1))))
        most = int(rng.integers(1, 32 // R + 1))
        yield L, R, Hkv, int(rng.choice([64, 128])), min(batch, MOST), most, int(np.exp(rng.uniform(np.log(500), np.log(1 << 30))))


def most_used(length, pairs, workgroups, start=START):
    """The most workgroups that lengths up to a bound give shares to: all, or one for every kLeastShare positions."""
    return min(workgroups, -(-pairs * (-(-length // 32) + start) // LEAST))


def test_the_most_parts_fit_the_workspace():
    shares, tight = 0, 0
    for L, R, Hkv, d, batch, most, length in cases():
        p = P.plan_of(L, R * Hkv, Hkv, d, batch, most, length)
        if p.chunk != 0:
            continue
        case = (L, R, Hkv, d, batch, most, length)
        every, _, at_bound = division([length] * batch, L * Hkv, p.chunks)
        used = most_used(length, L * Hkv * batch, p.chunks)
        assert every < 1 << 31 and at_bound <= used, case
        assert 2 * used <= slots_that_fit(p, d), case
        shares += 1
        tight += p.tiles == 2 and 2 * used + 2 >= slots_that_fit(p, d)
    assert shares > 5000 and tight > 1000


def test_a_workspace_for_shorter_starts_would_not_do():
    """What the test above is for: a bound that counts 4 blocks for a pair's start is too small for some of its cases."""
    small = 0
    for L, R, Hkv, d, batch, most, length in cases():
        p = P.plan_of(L, R * Hkv, Hkv, d, batch, most, length)
        if p.chunk != 0 or p.tiles != 2:
            continue
        heads = L * Hkv * batch
        chunks = min(heads * R * most * -(-length // 512), 64 * 8 * 256 + 32 * heads * -(-length // 4096))  # rows of cache_plan
        short = max(64 * min(256, heads * (-(-length // 32) + 4) // LEAST + 1), chunks)
        small += 64 * most_used(length, heads, p.chunks) > short
    assert small > 100


@pytest.mark.parametrize("heads", [(1, 1, 64), (2, 8, 4), (32, 2, 1), (1, 8, 1000)])
def test_positions_stay_below_two_to_the_31(heads):
    """The longest bound that is divided, and the next: a block more for every pair would pass 2^31."""
    L, Hkv, batch = heads
    blocks = ((1 << 31) - 1) // (L * Hkv * batch) - START
    for more, divided in ((0, True), (1, False)):
        p = P.plan_of(L, Hkv, Hkv, 64, batch, 1, min((blocks + more) * 32, (1 << 30)))
        assert (p.chunk == 0) == divided, (heads, more)
    assert L * Hkv * batch * (blocks + START) < 1 << 31 <= L * Hkv * batch * (blocks + 1 + START)
