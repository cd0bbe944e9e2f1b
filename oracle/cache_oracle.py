"""CPU oracle of the paged 4-bit cache (include/taskpress.h): test infrastructure only.

Plain float64 definitions, one token or one row at a time, and the bytes of a block by the documented
places of a code.  Rows are bf16 values given as float64; pages are a numpy byte array
[L][num_pages][Hkv][page_tokens / 32][block bytes]."""
from __future__ import annotations

import math

import numpy as np

BLOCK = 32  # tokens
HALVES, PAIRS = 0, 1
_MAX_BF16 = float(np.uint32(0x7F7F0000).view(np.float32))


def block_bytes(d):
    return BLOCK * (d + d // 16 + 4)


def to_bf16(x):
    """float64 -> the nearest bf16 value (ties to even), as float64; beyond the largest finite one, that one."""
    x = np.clip(np.asarray(x, dtype=np.float64), -_MAX_BF16, _MAX_BF16)
    unit = np.exp2(np.maximum(np.frexp(x)[1], -125) - 8.0)  # of the last of 8 significant bits; 2^-133 below 2^-126
    return np.rint(x / unit) * unit


def by_fp32(x):
    """float64 -> the nearest fp32 value -> the nearest bf16 value, as float64."""
    return to_bf16(np.clip(x, -_MAX_BF16, _MAX_BF16).astype(np.float32))


def bf16_bits(x):
    return (np.asarray(x, dtype=np.float64).astype(np.float32).view(np.uint32) >> 16).astype(np.uint16)


def rotate(x, cos_sin_row, rotary_dim, style):
    """One row [d], rotated by the angles of a table row [rotary_dim] (cosines, then sines)."""
    x, out = np.asarray(x, dtype=np.float64), np.array(x, dtype=np.float64)
    h = rotary_dim // 2
    for i in range(h):
        a, b = (i, i + h) if style == HALVES else (2 * i, 2 * i + 1)
        c, s = float(cos_sin_row[i]), float(cos_sin_row[h + i])
        out[a], out[b] = x[a] * c - x[b] * s, x[b] * c + x[a] * s
    return by_fp32(out)


def quantise_key(k):
    """One bf16 row [d]: codes int [d], scales float64 [d / 32] (bf16 values)."""
    codes, scales = [], []
    for i in range(0, len(k), 32):
        x = np.asarray(k[i:i + 32], dtype=np.float64)
        g = float(to_bf16(np.abs(x).max() / 7.0))
        codes.append(np.clip(np.rint(x / g), -7, 7) if g > 0 else np.zeros(32))
        scales.append(g)
    return np.concatenate(codes).astype(int), np.array(scales)


def quantise_value(v):
    """One bf16 row [d]: codes int [d] and the fp32 scale, Eq. 2 at bits = 4."""
    v = np.asarray(v, dtype=np.float64)
    g = np.float32(np.abs(v).max() / 7.0)
    if g == 0:
        return np.zeros(len(v), dtype=int), g
    return np.clip(np.rint((v / np.float64(g)).astype(np.float32)), -7, 7).astype(int), g


def _nibble(e):
    return e // 2 + 4 * (e % 2)


def key_place(d, token, channel):
    """(byte, shift) of a key's code in its block."""
    s, h, e = channel // 32, channel % 32 // 8, channel % 8
    word = token * (d // 8) + h * (d // 32) + s
    return 4 * word + _nibble(e) // 2, 4 * (_nibble(e) % 2)


def value_place(d, token, channel):
    g, e = token % 16 // 4, token // 16 * 4 + token % 4
    word = channel // 64 * 256 + (16 * g + channel % 16) * 4 + channel // 16 % 4
    return 16 * d + 4 * word + _nibble(e) // 2, 4 * (_nibble(e) % 2)


_places = {}


def places(d):
    """Bytes and shifts of all keys' and values' codes of a block: four arrays [32][d]."""
    if d not in _places:
        k = np.array([[key_place(d, t, c) for c in range(d)] for t in range(BLOCK)])
        v = np.array([[value_place(d, t, c) for c in range(d)] for t in range(BLOCK)])
        _places[d] = k[..., 0], k[..., 1], v[..., 0], v[..., 1]
    return _places[d]


def write_token(block, d, slot, key, value):
    """block: uint8 [bytes], changed in place; key = (codes, scales), value = (codes, scale)."""
    kb, ks, vb, vs = places(d)
    for at, shift, codes in ((kb[slot], ks[slot], key[0]), (vb[slot], vs[slot], value[0])):
        for b, s, c in zip(at, shift, codes):
            block[b] = block[b] & ~(15 << s) & 0xFF | (int(c) + 8) << s
    n = d // 32
    block[32 * d + 2 * n * slot:32 * d + 2 * n * (slot + 1)] = bf16_bits(key[1]).view(np.uint8)
    block[34 * d + 4 * slot:34 * d + 4 * slot + 4] = np.array([value[1]], dtype=np.float32).view(np.uint8)


def read_block(block, d):
    """The keys and values a block stands for, float64 [32][d] each."""
    kb, ks, vb, vs = places(d)
    k = (block[kb] >> ks & 15).astype(np.float64) - 8
    v = (block[vb] >> vs & 15).astype(np.float64) - 8
    bits = block[32 * d:34 * d].copy().view(np.uint16).astype(np.uint32) << 16
    k *= np.repeat(bits.view(np.float32).astype(np.float64).reshape(BLOCK, d // 32), 32, axis=1)
    return k, v * block[34 * d:].copy().view(np.float32).astype(np.float64)[:, None]


def place_of(table_row, num_pages, page_tokens, token):
    """(page, block of the page, slot) of a token, or None where it has no page."""
    page = int(table_row[token // page_tokens])
    if not 0 <= page < num_pages:
        return None
    return page, token % page_tokens // BLOCK, token % BLOCK


def held(pages, d, table_row, page_tokens, layer, head, n):
    """Keys and values of tokens 0..n-1 of a sequence, float64 [n][d], and whether each has a page."""
    k, v, there = np.zeros((n, d)), np.zeros((n, d)), np.zeros(n, dtype=bool)
    for t in range(0, n, BLOCK):
        at = place_of(table_row, pages.shape[1], page_tokens, t)
        if at is None:
            continue
        m = min(BLOCK, n - t)
        kk, vv = read_block(pages[layer, at[0], head, at[1]], d)
        k[t:t + m], v[t:t + m], there[t:t + m] = kk[:m], vv[:m], True
    return k, v, there


def attend(q, k, v, visible, scale):
    """One query row over the keys that `visible` marks: output [d], log-sum-exp, and the mean of |v| under the
    same weights (what errors of the weights are measured by)."""
    if not visible.any():
        return np.zeros(len(q)), -math.inf, np.zeros(len(q))
    x = scale * (k[visible] @ q)
    m = x.max()
    p = np.exp(x - m)
    z = p.sum()
    return p @ v[visible] / z, m + math.log(z), p @ np.abs(v[visible]) / z
