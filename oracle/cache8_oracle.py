"""CPU oracle of the paged 8-bit cache (include/taskpress.h): test infrastructure only.

Plain float64 definitions of a block's bytes by the documented places of a code; rotation, page lookup and attention
are cache_oracle's.  Rows are bf16 values given as float64; pages are a numpy byte array
[L][num_pages][Hkv][page_tokens / 32][block bytes]."""
from __future__ import annotations

import numpy as np

from oracle import taskpress_oracle as o
from oracle.cache_oracle import BLOCK, place_of

INT, FP8 = o.QFMT_INT, o.QFMT_FP8_E4M3


def block_bytes(d):
    return 64 * d + 144


def qmax(fmt):
    return 448.0 if fmt == FP8 else 127.0


def bytes_of(y, fmt):
    """Bytes of the codes nearest to numbers y."""
    y = np.asarray(y, dtype=np.float64)
    return o.e4m3_encode(y) if fmt == FP8 else (np.clip(np.rint(y), -127, 127) + 128).astype(np.uint8)


def codes_of(b, fmt):
    """The numbers that bytes stand for (float64)."""
    return o.e4m3_decode(b) if fmt == FP8 else b.astype(np.float64) - 128


def quantised(x, scale, fmt):
    """Bytes of rows x in an fp32 scale: codes of fl32(x / scale), 0 where the scale is 0."""
    s = np.float64(scale)
    y = np.where(s > 0, (np.asarray(x, dtype=np.float64) / np.where(s > 0, s, 1.0)).astype(np.float32), np.float32(0))
    return bytes_of(y, fmt)


def key_place(d, token, x):
    return token // 16 * 16 * d + x // 64 * 1024 + (x % 32 // 8 * 16 + token % 16) * 16 + x // 32 % 2 * 8 + x % 8


def value_place(d, token, x):
    return 32 * d + x // 32 * 1024 + (token % 16 // 4 * 16 + x % 16) * 16 + x // 16 % 2 * 8 + token // 16 * 4 + token % 4


_places = {}


def places(d):
    """Bytes of all keys' and values' codes of a block: two arrays [32][d]."""
    if d not in _places:
        _places[d] = tuple(np.array([[f(d, t, x) for x in range(d)] for t in range(BLOCK)]) for f in (key_place, value_place))
    return _places[d]


def key_scale(block, d):
    return block[64 * d + 128:64 * d + 132].copy().view(np.float32)[0]


def write_keys(block, d, fmt, before, keys):
    """keys: {slot: row} that one call writes; before: the tokens of the block before the call's first."""
    if not keys:
        return
    at = places(d)[0]
    m = max(np.abs(k).max() for k in keys.values())
    want = np.float32(m / qmax(fmt))
    held = key_scale(block, d) if before > 0 else np.float32(0)
    scale = want
    if 0 < held < np.inf:
        n = 0
        while float(held) * 2.0 ** n < float(want):
            n += 1
        scale = np.float32(float(held) * 2.0 ** n)
        if n:
            for t in range(before):
                block[at[t]] = bytes_of(codes_of(block[at[t]], fmt) * 2.0 ** -n, fmt)
    block[64 * d + 128:64 * d + 132] = np.array([scale], dtype=np.float32).view(np.uint8)
    for slot, k in keys.items():
        block[at[slot]] = quantised(k, scale, fmt)


def write_value(block, d, slot, value_bytes, scale):
    block[places(d)[1][slot]] = value_bytes
    block[64 * d + 4 * slot:64 * d + 4 * slot + 4] = np.array([scale], dtype=np.float32).view(np.uint8)


def quantise_value(v, fmt):
    """One bf16 row [d]: bytes [d] and the fp32 scale (Eq. 2)."""
    g = np.float32(np.abs(v).max() / qmax(fmt))
    return quantised(v, g, fmt), g


def read_block(block, d, fmt):
    """The keys and values a block stands for, float64 [32][d] each."""
    k, v = (codes_of(block[at], fmt) for at in places(d))
    return k * np.float64(key_scale(block, d)), v * block[64 * d:64 * d + 128].copy().view(np.float32).astype(np.float64)[:, None]


def held(pages, d, fmt, table_row, page_tokens, layer, head, n):
    """Keys and values of tokens 0..n-1 of a sequence, float64 [n][d], and whether each has a page."""
    k, v, there = np.zeros((n, d)), np.zeros((n, d)), np.zeros(n, dtype=bool)
    for t in range(0, n, BLOCK):
        at = place_of(table_row, pages.shape[1], page_tokens, t)
        if at is None:
            continue
        m = min(BLOCK, n - t)
        kk, vv = read_block(pages[layer, at[0], head, at[1]], d, fmt)
        k[t:t + m], v[t:t + m], there[t:t + m] = kk[:m], vv[:m], True
    return k, v, there
