"""Contents of a paged cache on which a wrong attention shows, and how far a right one may be off, row by row.

A row's error, from the kernel's arithmetic (all first-order terms are kept, e is what a weight may be off):
  score    d products of a code times its scale and a query, exact, summed in fp32 in some order, the sum perhaps
           truncated: (d + 8) 2^-23 sum |k_i q_i| scale, and 2^-22 |x| for the factor log2(e) and the exponent's
           argument; 2^-21 for exp2 itself;
  weight   its product with the value's scale in fp16, 2^-11, or within 2^-25 of a number at least 2^8 where it is more
           than 2^22 below the row's largest: 2^-10.9 sum p |v| + N 2^-30 max |v|;
  sums     2^-14 of the normaliser and of the output (a lane adds at most 512 numbers of a chunk, then 32 chunks);
  output   rounded to bf16: 2^-8 |o|."""
import math

import numpy as np

from oracle import cache_oracle as c


def bounds(q, k, v, visible, scale):
    """One row: output and log-sum-exp, and how far they may be off."""
    ref, lse, mag = c.attend(q, k, v, visible, scale)
    if not visible.any():
        return ref, lse, np.zeros(len(q)), 0.0
    kk, vv = k[visible], np.abs(v[visible])
    x = scale * (kk @ q)
    delta = scale * (len(q) + 8) * 2.0 ** -23 * (np.abs(kk) @ np.abs(q)) + 2.0 ** -22 * np.abs(x) + 2.0 ** -21
    e = np.exp(x - lse + delta) - np.exp(x - lse)
    total = e.sum()
    tol = (e @ vv + total * np.abs(ref) + mag * (2.0 ** -10.9 + 2.0 ** -14) + 2.0 ** -8 * np.abs(ref)
           + len(v) * 2.0 ** -30 * np.abs(v).max())
    return ref, lse, tol, math.log1p(total) + 2.0 ** -14 + 2.0 ** -22 * abs(lse)


def accepts(o, lse, bound):
    ref, want, tol, tol_lse = bound
    if want == -math.inf:
        return lse == -math.inf and not np.any(o)
    return bool(np.all(np.abs(o - ref) <= tol)) and abs(lse - want) <= tol_lse


def rows(s, new, q, scale, only=None):
    """The bounds of every row of a setup (test_gpu_cache.Setup), one layer: (token row, query head, bound)."""
    off, R = np.concatenate([[0], np.cumsum(new)]), s.Hq // s.Hkv
    for b in only or range(len(new)):
        n = s.lens_[b]
        for h in range(s.Hkv):
            k, v, there = c.held(s.pages, s.d, s.table[b], s.page, 0, h, n)
            for t in range(new[b]):
                visible = there & (np.arange(n) <= n - new[b] + t)
                for hq in range(h * R, (h + 1) * R):
                    yield off[b] + t, hq, bounds(q[0, off[b] + t, hq], k, v, visible, scale)


KINDS = ["ordinary", "powers", "weak", "levels", "massive", "peaked", "far"]


def fill(s, kind, n):
    """Writes the kind's key codes and scales into a setup's pages (its values stay), and returns queries of n new tokens
    and the factor of the scores.  Scores are of order 1 unless the kind says otherwise."""
    rng, d = s.rng, s.d
    G = d // 32
    blocks = s.pages.reshape(-1, c.block_bytes(d))
    words = blocks[:, :16 * d].reshape(len(blocks), 32, 4, G, 4)  # [token][h][group]: channels 32 group + 8 h + 0..7
    ks = rng.uniform(0.1, 0.5, (len(blocks), 32, G))
    q, scale = c.to_bf16(rng.normal(size=(1, n, s.Hq, d)) * 1.5), 1 / math.sqrt(d)
    if kind in ("powers", "weak", "levels"):
        # group 0 is stronger, by another power of two from block to block; the queries leave it out, so the others decide
        q[..., :32] = 0
        if kind == "powers":    # within what one power of two for all groups holds
            ks[..., 0] *= 2.0 ** rng.integers(-4, 17, (len(blocks), 1))
        elif kind == "weak":    # beyond it in most blocks
            ks[..., 0] *= 2.0 ** rng.integers(10, 100, (len(blocks), 1))
        else:  # three levels more (d = 128); what a group's keys lack its queries make up for, up to 2^22 (there they are exact)
            ks[..., 0] *= 2.0 ** 45
            ks[..., 1:] *= 2.0 ** np.array([0, -13, -26])[:G - 1]
            q[..., 32:] *= np.repeat(2.0 ** np.array([0, 13, 22])[:G - 1], 32)
        ks[rng.random(ks.shape[:2]) < 0.05] = 0  # some keys are zero
    elif kind == "massive":
        # some blocks have a token whose score is far below the others', which must not lose theirs
        q[..., 0] = 4.0
        for i in range(0, len(blocks), 2):
            t = rng.integers(32)
            words[i, t] = 0x88       # codes 0
            words[i, t, 0, 0, 0] = 0x81  # channel 0: -7
            ks[i, t] *= 2.0 ** rng.integers(15, 40)
    elif kind == "peaked":
        q = c.to_bf16(q * 4)
    elif kind == "far":
        # scores of 1000 and what the other channels add
        ks[..., 0] = 0.25
        words[:, :, 0, 0, 0] |= 0x0F  # channel 0: 7
        q[..., 0] = float(c.to_bf16(1000 * math.sqrt(d) / 1.75))
    blocks[:, 32 * d:34 * d] = c.bf16_bits(ks.reshape(len(blocks), -1)).view(np.uint8).reshape(len(blocks), -1)
    return q, scale


# (query heads, KV heads, lengths, new tokens, length bound): 16 rows and fewer in eight and in four waves, then two and
# four tiles of 16, sequences whole and in chunks; a wave's blocks are several
SHAPES = [(8, 2, [960, 95], [1, 1], 960), (8, 2, [2100, 300], [1, 2], 2100), (8, 2, [960, 95], [5, 3], 960),
          (8, 2, [2100, 300], [6, 1], 2100), (8, 2, [700, 95], [9, 2], 700), (8, 2, [2100, 31], [10, 16], 2100)]
