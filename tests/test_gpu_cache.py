"""The paged 4-bit cache through the C ABI on the GPU, against the float64 oracle.

What is written is compared byte for byte over the whole pool, so what a call must leave alone is checked
too.  Attention's tolerances, per output element, from its arithmetic:
  weights   a weight times its value's scale is rounded to fp16 (half a step: 2^-11), or, more than 2^22
            below the row's largest, held within 2^-25 of a number at least 2^8: together at most
            2^-11 sum p |v| + N 2^-33 7 max(p scale) <= 2^-10.9 sum p |v| + N 2^-30 max |v|;
  scores    a group's product has 32 terms of at most 7 |q|, summed in fp32 in some order, and then up to four groups'
            sums times their scales: an error of at most delta = scale * sum over groups of (max key scale)
            * 72 * 2^-24 * 7 * sum |q| (32 for the terms, 8 for the groups, and 32 = 2^-19 * 2^24 for a scale
            so far below its block's largest that it counts as zero) + 2^-22 max |x| (the factor log2(e), the exponent's
            argument), and 2^-21 for exp2 itself; a weight is off by that share, twice with the normaliser:
            2 (delta + 2^-21) sum p |v|;
  sums      a lane adds at most 512 p's of a chunk, 32 chunks: 2^-14 of the normaliser, 2^-14 of the output;
  output    rounded to bf16: 2^-8 |o|.
The log-sum-exp, fp32: delta + 2^-14 + 2^-22 |lse|."""
import math

import numpy as np
import pytest
import torch

from oracle import cache_oracle as c
from oracle import taskpress_oracle as o
from paper_2608_03276_amd import binding as B

pytestmark = pytest.mark.gpu


def bf16(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(torch.bfloat16)


def f64(t):
    return t.detach().double().cpu().numpy()


class Setup:
    """A cache of random contents with shuffled pages, on the host and on the GPU."""

    def __init__(self, seed, L, Hq, Hkv, d, page, lens, cols=None, spare=2, fill=True):
        self.rng = np.random.default_rng(seed)
        self.L, self.Hq, self.Hkv, self.d, self.page, self.lens_ = L, Hq, Hkv, d, page, list(lens)
        self.dims = B.dims(L, Hq, Hkv, d)
        need = [-(-max(n, 0) // page) for n in lens]
        self.num = sum(need) + spare
        order = self.rng.permutation(self.num)
        self.table = np.full((len(lens), cols or max(max(need), 1)), -1, dtype=np.int32)
        i = 0
        for b, n in enumerate(need):
            self.table[b, :n] = order[i:i + n]
            i += n
        self.pages = self.rng.integers(0, 256, (L, self.num, Hkv, page // 32, c.block_bytes(d))).astype(np.uint8)
        if fill:  # finite scales of ordinary keys and values
            blocks = self.pages.reshape(-1, c.block_bytes(d))
            blocks[:, 32 * d:34 * d] = c.bf16_bits(self.rng.uniform(0.1, 0.5, (len(blocks), d))).view(np.uint8).reshape(len(blocks), -1)
            vs = (self.rng.uniform(0.1, 0.5, (len(blocks), 32)) * np.where(self.rng.random((len(blocks), 32)) < 0.05, 20, 1))
            blocks[:, 34 * d:] = vs.astype(np.float32).view(np.uint8).reshape(len(blocks), -1)
        self.upload()

    def upload(self):
        self.dev = torch.from_numpy(self.pages.copy()).cuda()
        self.lens = torch.tensor(self.lens_, dtype=torch.int32, device="cuda")
        self.dtable = torch.from_numpy(self.table.copy()).cuda()
        self.cache = B.Cache(self.dims, self.dev, self.dtable, self.lens, self.page)

    def rows(self, n, heads, scale=1.0):
        return c.to_bf16(self.rng.normal(size=(self.L, n, heads, self.d)) * scale)

    def write(self, b, token, layer, head, key, value):
        at = c.place_of(self.table[b], self.num, self.page, token)
        if at is not None:
            c.write_token(self.pages[layer, at[0], head, at[1]], self.d, at[2], key, value)

    def check_pages(self):
        got = self.dev.cpu().numpy()
        if not np.array_equal(got, self.pages):
            bad = np.argwhere(got != self.pages)
            raise AssertionError(f"{len(bad)} bytes differ, first at {bad[0]} (block bytes {c.block_bytes(self.d)})")


def same(got, want):
    if not np.array_equal(got, want):
        at = tuple(np.argwhere(got != want)[0])
        raise AssertionError(f"{int((got != want).sum())} of {got.size} differ, first at {at}: {got[at]!r}, expected {want[at]!r}")


def table_of(positions, r, theta=10000.0):
    freq = theta ** (-np.arange(0, r, 2) / r)
    a = np.arange(positions)[:, None] * freq
    return np.concatenate([np.cos(a), np.sin(a)], 1).astype(np.float32)


def offsets_of(new):
    return np.concatenate([[0], np.cumsum(new)]).astype(np.int32)


# ------------------------------------------------------------------------------ append
APPENDS = [
    # (L, Hq, Hkv, d, page, lens, new, rotary_dim (0: none), style, with q)
    (1, 8, 2, 64, 32, [1, 33, 64, 257], [1, 1, 1, 1], 64, 0, True),
    (1, 8, 2, 128, 64, [1, 32, 65, 300], [1, 1, 1, 1], 128, 0, True),
    (2, 12, 4, 64, 64, [40, 0, 129, 5], [40, 0, 70, 3], 64, 1, True),
    (1, 5, 5, 128, 256, [300, 31, 512], [259, 7, 1], 128, 1, True),
    (1, 4, 1, 128, 128, [7, 200], [7, 33], 32, 0, True),       # some channels rotated
    (2, 16, 2, 64, 32, [95, 64], [40, 64], 48, 1, True),
    (1, 8, 2, 128, 32, [50, 3], [17, 3], 0, 0, False),         # no rotation
    (1, 64, 8, 128, 64, [70], [70], 128, 0, True),
]


@pytest.mark.parametrize("case", APPENDS, ids=[f"L{a[0]}h{a[1]}-{a[2]}d{a[3]}p{a[4]}r{a[7]}s{a[8]}" for a in APPENDS])
def test_append(gpu_lib, case):
    L, Hq, Hkv, d, page, lens, new, r, style, with_q = case
    s = Setup(11, L, Hq, Hkv, d, page, lens)
    n, off = sum(new), offsets_of(new)
    total = n + 2  # padded: two rows of no sequence
    k, v, q = (s.rows(total, h) for h in (Hkv, Hkv, Hq))
    v[0, 0, 0] = 0.0
    k[0, 0, 0, :32] = 0.0
    cs = table_of(500, r) if r else None
    pos = s.rng.integers(0, 500, total).astype(np.int32)
    q_dev = bf16(q).cuda()
    q_out = torch.full_like(q_dev, -7.0)
    step = B.Step(total, max(new), torch.from_numpy(off).cuda())
    kw = dict(positions=torch.from_numpy(pos).cuda(), rope=B.Rope(torch.from_numpy(cs).cuda(), r, style)) if r else {}
    if with_q:
        kw.update(q=q_dev, q_out=q_out)
    B.tp_cache_append(s.dims, s.cache, step, bf16(k).cuda(), bf16(v).cuda(), **kw)
    torch.cuda.synchronize()
    want = np.full(q.shape, -7.0)
    for b in range(len(lens)):
        for t in range(new[b]):
            row = off[b] + t
            turn = (lambda x: c.rotate(x, cs[pos[row]], r, style)) if r else (lambda x: x)
            for l in range(L):
                for h in range(Hkv):
                    s.write(b, lens[b] - new[b] + t, l, h, c.quantise_key(turn(k[l, row, h])), c.quantise_value(v[l, row, h]))
                for h in range(Hq):
                    want[l, row, h] = turn(q[l, row, h])
    s.check_pages()
    same(f64(q_out), want if with_q else np.full(q.shape, -7.0))


@pytest.mark.parametrize("d", [64, 128])
def test_append_odd_values(gpu_lib, d):
    """Keys and values at the edges of the format: ties, the smallest and largest numbers, one-sided rows."""
    s = Setup(12, 1, 2, 2, d, 32, [32])
    k, v = s.rows(32, 2), s.rows(32, 2)
    for t, scale in enumerate([2.0 ** -133, 3 * 2.0 ** -133, 2.0 ** -126, 2.0 ** -100, 2.0 ** -60, 2.0 ** 60, 2.0 ** 100, 2.0 ** 125]):
        k[0, t], v[0, t] = c.to_bf16(k[0, t] / 8 * scale), c.to_bf16(v[0, t] / 8 * scale)
    k[0, 8] = v[0, 8] = c.to_bf16(s.rng.integers(-14, 15, (2, d)) / 2)  # absmax 7 in most groups: ties
    k[0, 8, :, ::32] = v[0, 8, :, ::32] = 7.0
    k[0, 9] = v[0, 9] = c._MAX_BF16
    k[0, 10] = v[0, 10] = -c._MAX_BF16
    for t in range(11, 32):  # every code's border, at scales of all significands
        g = float(c.to_bf16(1 + s.rng.integers(0, 128, (2, d // 32)) / 128)[0, 0])
        k[0, t] = c.to_bf16(g * (s.rng.integers(-7, 7, (2, d)) + 0.5 + s.rng.choice([-1, 0, 1], (2, d)) * 2.0 ** -8))
        k[0, t, :, ::32] = c.to_bf16(7 * g)
    step = B.Step(32, 32, torch.tensor([0, 32], dtype=torch.int32, device="cuda"))
    B.tp_cache_append(s.dims, s.cache, step, bf16(k).cuda(), bf16(v).cuda())
    for t in range(32):
        for h in range(2):
            s.write(0, t, 0, h, c.quantise_key(k[0, t, h]), c.quantise_value(v[0, t, h]))
    s.check_pages()


def test_append_rotation_saturates(gpu_lib):
    s = Setup(13, 1, 1, 1, 64, 32, [1])
    k = np.full((1, 1, 1, 64), c._MAX_BF16)
    cs = np.concatenate([np.full(32, 0.8), np.full(32, 0.6)]).astype(np.float32)[None]
    q_out = torch.zeros((1, 1, 64), dtype=torch.bfloat16, device="cuda")
    B.tp_cache_append(s.dims, s.cache, B.Step(1), bf16(k).cuda(), bf16(k).cuda(), torch.zeros(1, dtype=torch.int32, device="cuda"),
                      B.Rope(torch.from_numpy(cs).cuda(), 64), bf16(k[0]).cuda(), q_out)
    key = c.rotate(k[0, 0, 0], cs[0], 64, 0)
    assert key[32] == c._MAX_BF16
    s.write(0, 0, 0, 0, c.quantise_key(key), c.quantise_value(k[0, 0, 0]))
    s.check_pages()
    same(f64(q_out)[0, 0], key)


def test_append_leaves_out_what_is_out_of_range(gpu_lib):
    """Lengths, offsets, pages and positions that no token has: nothing is written for them."""
    new = [2, 2, 3, 2, 2, 2, 5]
    lens = [40, 41, 2, 64, 1000, -5, 64]  # 2 < 3 new: the first is before the start; 1000 and -5 count as 0
    s = Setup(14, 1, 4, 2, 64, 32, [min(max(n, 0), 64) for n in lens], cols=2)
    s.table[1, 1], s.table[3, 1] = -1, s.num  # the pages of sequences 1's and 3's newest tokens
    s.lens_ = lens
    s.upload()
    off = offsets_of(new)
    total = int(off[-1])
    k, v, q = s.rows(total, 2), s.rows(total, 2), s.rows(total, 4)
    cs = table_of(50, 64)
    pos = s.rng.integers(0, 50, total).astype(np.int32)
    pos[0], pos[5] = 50, -1  # sequence 0's first, sequence 2's second token
    q_out = torch.full((total, 4, 64), -7.0, dtype=torch.bfloat16, device="cuda")
    step = B.Step(total, 3, torch.from_numpy(off).cuda())  # sequence 6 has more than 3: none
    B.tp_cache_append(s.dims, s.cache, step, bf16(k).cuda(), bf16(v).cuda(), torch.from_numpy(pos).cuda(),
                      B.Rope(torch.from_numpy(cs).cuda(), 64), bf16(q[0]).cuda(), q_out)
    want = np.full((total, 4, 64), -7.0)
    for b in range(7):
        for t in range(new[b]):
            row, token = off[b] + t, lens[b] - new[b] + t
            if new[b] > 3 or not 0 <= pos[row] < 50:
                continue
            for h in range(4):
                want[row, h] = c.rotate(q[0, row, h], cs[pos[row]], 64, 0)
            if 0 <= token < 64 and 0 <= lens[b] <= 64:
                for h in range(2):
                    s.write(b, token, 0, h, c.quantise_key(c.rotate(k[0, row, h], cs[pos[row]], 64, 0)), c.quantise_value(v[0, row, h]))
    s.check_pages()
    same(f64(q_out), want)


@pytest.mark.parametrize("bad", [[0, 3, 2, 5], [0, 2, 9, 5], [-1, 2, 4, 5], [3, 4, 5, 6]])
def test_append_bad_offsets(gpu_lib, bad):
    """Ranges that decrease or leave the tensors count as empty; the others are written."""
    s = Setup(15, 1, 2, 1, 64, 32, [30, 31, 32])
    k, v = s.rows(5, 1), s.rows(5, 1)
    q = s.rows(5, 2)
    q_out = torch.full((5, 2, 64), -7.0, dtype=torch.bfloat16, device="cuda")
    cs, pos = table_of(9, 64), np.arange(5).astype(np.int32)
    B.tp_cache_append(s.dims, s.cache, B.Step(5, 4, torch.tensor(bad, dtype=torch.int32, device="cuda")), bf16(k).cuda(),
                      bf16(v).cuda(), torch.from_numpy(pos).cuda(), B.Rope(torch.from_numpy(cs).cuda(), 64), bf16(q[0]).cuda(), q_out)
    good = set()
    for b in range(3):
        lo, hi = bad[b], bad[b + 1]
        if lo < 0 or hi > 5 or hi <= lo:
            continue
        for t in range(hi - lo):
            good.add(lo + t)
            s.write(b, s.lens_[b] - (hi - lo) + t, 0, 0, c.quantise_key(c.rotate(k[0, lo + t, 0], cs[lo + t], 64, 0)),
                    c.quantise_value(v[0, lo + t, 0]))
    s.check_pages()
    got = f64(q_out)
    for row in range(5):
        if row not in good:  # rows of no sequence are left alone
            assert np.all(got[row] == -7.0)


# ------------------------------------------------------------------------------ load and read
@pytest.mark.parametrize("bits", [2, 3, 4])
@pytest.mark.parametrize("L,Hkv,d,page,kept", [(2, 2, 64, 32, [70, 0, 32, 1]), (1, 3, 128, 128, [129, 31]), (3, 1, 128, 64, [5])])
def test_load(gpu_lib, bits, L, Hkv, d, page, kept):
    s = Setup(21, L, Hkv, Hkv, d, page, kept)
    n = sum(kept)
    k = c.to_bf16(s.rng.normal(size=(L, Hkv, n, d)))
    v = bf16(s.rng.standard_t(3, size=(L, Hkv, n, d))).cuda()
    scales = torch.empty((L, Hkv, n), device="cuda")
    v_q = torch.empty((L, Hkv, n, d // 2), dtype=torch.uint8, device="cuda")
    B.tp_quantize_v_scales(s.dims, B.Batch([0, n]), v, B.TP_QFMT_INT, bits, scales, v_q)
    off = offsets_of(kept).tolist()
    B.tp_cache_load(s.dims, s.cache, off, bf16(k).cuda(), v_q, scales, bits)
    vv = f64(v)
    for b in range(len(kept)):
        for t in range(kept[b]):
            for l in range(L):
                for h in range(Hkv):
                    row = vv[l, h, off[b] + t]
                    g = o.value_scales(row[None], o.QFMT_INT, bits)
                    s.write(b, t, l, h, c.quantise_key(k[l, h, off[b] + t]), (o.quantize_values(row[None], g, o.QFMT_INT, bits)[0], g[0]))
    s.check_pages()


@pytest.mark.parametrize("d,page", [(64, 32), (128, 64), (128, 256)])
def test_read(gpu_lib, d, page):
    lens = [300, 5, 64, 0, 128]
    s = Setup(22, 2, 2, 2, d, page, lens, spare=3)
    s.table[2, 0] = -3  # a sequence whose first page is missing
    s.lens_[4] = 90     # fewer tokens than its pages hold
    s.upload()
    first, count = [37, 0, 0, 0, 60], [263, 9, 64, 3, 68]
    off = offsets_of(count).tolist()
    k = torch.full((2, 2, off[-1], d), -7.0, dtype=torch.bfloat16, device="cuda")
    v = torch.full_like(k, -7.0)
    B.tp_cache_read(s.dims, s.cache, B.Batch(off), k, v, first)
    for b in range(5):
        for l in range(2):
            for h in range(2):
                kk, vv, _ = c.held(s.pages, d, s.table[b], page, l, h, s.lens_[b])
                want = np.zeros((2, count[b], d))
                m = max(0, min(s.lens_[b] - first[b], count[b]))
                want[0, :m], want[1, :m] = kk[first[b]:first[b] + m], vv[first[b]:first[b] + m]
                want = c.by_fp32(want)
                same(f64(k[l, h, off[b]:off[b + 1]]), want[0]), (b, l, h)
                same(f64(v[l, h, off[b]:off[b + 1]]), want[1]), (b, l, h)
    # from the start
    B.tp_cache_read(s.dims, s.cache, B.Batch(off), k, v)
    kk, vv, _ = c.held(s.pages, d, s.table[0], page, 1, 1, 263)
    same(f64(k[1, 1, :263]), c.by_fp32(kk))
    same(f64(v[1, 1, :263]), c.by_fp32(vv))


@pytest.mark.parametrize("d", [64, 128])
def test_read_more_than_the_caches_hold(gpu_lib, d):
    """Outputs above 256 MB (streaming stores): the same rows, zeros behind the sequences, rows outside the ranges kept."""
    s = Setup(23, 1, 8, 8, d, 64, [300, 97])
    few = torch.empty((8, 397, d), dtype=torch.bfloat16, device="cuda")
    fewv = torch.empty_like(few)
    B.tp_cache_read(s.dims, s.cache, B.Batch([0, 297, 397]), few, fewv, [3, 0])
    n = (1 << 28) // (8 * d * 4) + 333
    k = torch.full((1, 8, n, d), -7.0, dtype=torch.bfloat16, device="cuda")
    v = torch.full_like(k, -7.0)
    B.tp_cache_read(s.dims, s.cache, B.Batch([0, 297, n]), k, v, [3, 0])
    for got, want in ((k, few), (v, fewv)):
        assert torch.equal(got[0, :, :394], want[:, :394])
        assert not bool(got[0, :, 394:].any())


# ------------------------------------------------------------------------------ attention
@pytest.mark.parametrize("batch,off,total", [
    (4, [0, 1, 2, 0, 0], 3),                                     # unused entries behind the last sequence are 0
    (4, [0, 1, 2, -1, 0], 3),
    (5, [4, 5, 0, 1, 3, 3], 6),                                  # sequences out of order: row 3 belongs to none
    (200, list(range(150)) + [0] * 40 + [149, 151] + [7] * 9, 153),
    (200, [0] * 70 + list(range(131)), 140),
])
def test_append_queries_of_every_sequence(gpu_lib, batch, off, total):
    """Offsets that fall somewhere: the query rows of every range that counts are rotated, the others left alone."""
    assert len(off) == batch + 1
    s = Setup(19, 1, 2, 1, 64, 32, [5] * batch)
    k, v, q = s.rows(total, 1), s.rows(total, 1), s.rows(total, 2)
    cs, pos = table_of(9, 64), np.arange(total).astype(np.int32) % 9
    want = np.full((total, 2, 64), -7.0)
    for b in range(batch):
        lo, hi = off[b], off[b + 1]
        if lo < 0 or hi > total or hi <= lo or hi - lo > 3:
            continue
        for row in range(lo, hi):
            s.write(b, 5 - hi + row, 0, 0, c.quantise_key(c.rotate(k[0, row, 0], cs[pos[row]], 64, 0)), c.quantise_value(v[0, row, 0]))
            for h in range(2):
                want[row, h] = c.rotate(q[0, row, h], cs[pos[row]], 64, 0)
    q_out = torch.full((total, 2, 64), -7.0, dtype=torch.bfloat16, device="cuda")
    B.tp_cache_append(s.dims, s.cache, B.Step(total, 3, torch.tensor(off, dtype=torch.int32, device="cuda")), bf16(k).cuda(),
                      bf16(v).cuda(), torch.from_numpy(pos).cuda(), B.Rope(torch.from_numpy(cs).cuda(), 64), bf16(q[0]).cuda(), q_out)
    s.check_pages()
    same(f64(q_out), want)


def check_attention(s, q, new, got_o, got_lse, scale, only=None, heads=None):
    """q float64 [L][total][Hq][d]; got_o, got_lse as the call wrote them; returns the worst share of the tolerance.
    only: the sequences looked at (default: all), heads: the KV heads."""
    off, worst = offsets_of(new), 0.0
    R = s.Hq // s.Hkv
    cap = s.table.shape[1] * s.page
    for b in only or range(len(new)):
        n = s.lens_[b] if 0 <= s.lens_[b] <= cap else 0
        for l in range(s.L):
            for h in heads or range(s.Hkv):
                k, v, there = c.held(s.pages, s.d, s.table[b], s.page, l, h, n)
                seen_scale = np.abs(k).reshape(n, -1, 32).max(2).max(0) if n else np.zeros(s.d // 32)
                for t in range(new[b]):
                    row = off[b] + t
                    visible = there & (np.arange(n) <= n - new[b] + t)
                    for hq in range(h * R, (h + 1) * R):
                        ref, lse, mag = c.attend(q[l, row, hq], k, v, visible, scale)
                        gl = float(got_lse[l, hq, row])
                        go = got_o[l, row, hq]
                        tag = (b, l, hq, t)
                        if not visible.any():
                            assert gl == -math.inf and not go.any(), tag
                            continue
                        x = np.abs(scale * (k[visible] @ q[l, row, hq])).max()
                        # a group's scale is at most its largest |key| (some code is at least 1)
                        qs = np.abs(q[l, row, hq]).reshape(-1, 32).sum(1)
                        delta = scale * float((seen_scale * qs).sum()) * 72 * 7 * 2.0 ** -24 + 2.0 ** -22 * x
                        assert abs(gl - lse) <= delta + 2.0 ** -14 + 2.0 ** -22 * abs(lse), (tag, gl, lse)
                        tol = (mag * (2.0 ** -10.9 + 2 * (delta + 2.0 ** -21) + 2.0 ** -14) + 2.0 ** -8 * np.abs(ref)
                               + n * 2.0 ** -30 * np.abs(v).max())
                        err = np.abs(go - ref)
                        assert np.all(err <= tol), (tag, float((err / tol).max()))
                        worst = max(worst, float((err / np.maximum(tol, 1e-300)).max()))
    return worst


def attend(s, q, new, scale, max_len=None, total=None, max_new=None, lse=True, stream=None, ws=None):
    off = offsets_of(new)
    total = total or q.shape[1]
    step = B.Step(total, max_new or max(max(new), 1), torch.from_numpy(off).cuda())
    out = torch.full((s.L, total, s.Hq, s.d), -7.0, dtype=torch.bfloat16, device="cuda")
    l = torch.full((s.L, s.Hq, total), -7.0, device="cuda") if lse else None
    B.tp_cache_attention(s.dims, s.cache, step, bf16(q).cuda(), scale, max_len or s.table.shape[1] * s.page, out, l, ws, stream)
    torch.cuda.synchronize()
    return out, l


ATTENDS = [
    # (L, Hq, Hkv, d, page, lens, new)
    (1, 8, 2, 64, 32, [257], [1]),
    (1, 8, 2, 128, 64, [1, 31, 32, 33, 64, 127, 128, 129, 700], [1] * 9),
    (1, 32, 8, 128, 64, [1500, 3], [1, 1]),
    (2, 5, 5, 64, 128, [100, 0, 300], [1, 1, 1]),              # one query head a KV head, an empty sequence
    (1, 64, 2, 128, 256, [513], [1]),                          # 32 query heads a KV head
    (1, 8, 2, 128, 64, [40, 300, 9, 128], [5, 8, 9, 0]),       # drafted tokens; none for one sequence
    (1, 12, 4, 64, 32, [75, 7], [33, 9]),                      # more new tokens than held: rows that see nothing
    (1, 4, 1, 128, 32, [200], [90]),
    (1, 16, 1, 64, 64, [333, 64], [21, 64]),
    (1, 2, 2, 128, 128, [9000], [2]),                          # several chunks
    (1, 4, 1, 64, 32, [8193, 1], [1, 1]),
]


@pytest.mark.parametrize("case", ATTENDS, ids=[f"L{a[0]}h{a[1]}-{a[2]}d{a[3]}n{max(a[5])}t{max(a[6])}" for a in ATTENDS])
def test_attention(gpu_lib, case):
    L, Hq, Hkv, d, page, lens, new = case
    s = Setup(31, L, Hq, Hkv, d, page, lens)
    total = sum(new) + 1  # a row of no sequence
    q = s.rows(total, Hq, 1.5)
    out, lse = attend(s, q, new, 1 / math.sqrt(d))
    check_attention(s, q, new, f64(out), f64(lse), 1 / math.sqrt(d))
    assert bool((out[:, -1] == -7).all()) and bool((lse[:, :, -1] == -7).all())
    again, l2 = attend(s, q, new, 1 / math.sqrt(d))
    assert torch.equal(out, again) and torch.equal(lse, l2)
    alone, _ = attend(s, q, new, 1 / math.sqrt(d), lse=False)
    assert torch.equal(out, alone)


@pytest.mark.parametrize("d", [64, 128])
def test_attention_ignores_what_is_not_held(gpu_lib, d):
    """NaN and infinite scales in slots and pages beyond the sequences, missing pages, lengths that do not count."""
    lens = [37, 100, 64, 161, 50]
    s = Setup(32, 1, 4, 2, d, 32, lens, cols=6)
    nan16, nan32 = np.uint16(0x7FC0), np.float32(np.nan)
    for b, n in enumerate(lens):
        if n % 32:
            at = c.place_of(s.table[b], s.num, s.page, n - 1)
            for h in range(2):
                blk = s.pages[0, at[0], h, at[1]]
                blk[32 * d:34 * d].view(np.uint16).reshape(32, -1)[n % 32:] = nan16 if h else np.uint16(0x7F80)
                blk[34 * d:].view(np.float32)[n % 32:] = nan32 if h else np.inf
    s.table[1, 1] = -1          # tokens 32..63 of sequence 1
    s.table[2] = s.num + 5      # sequence 2 has no pages at all
    s.lens_[4] = 6 * 32 + 1     # beyond its pages: counts as empty
    s.upload()
    new = [2, 1, 1, 40, 1]
    q = s.rows(sum(new), 4)
    out, lse = attend(s, q, new, 0.2)
    check_attention(s, q, new, f64(out), f64(lse), 0.2)
    # a bound below a sequence's length empties that one only
    s.lens_[4] = 50
    s.upload()
    out, lse = attend(s, q, new, 0.2, max_len=128)
    s.lens_[3] = 10 ** 9
    check_attention(s, q, new, f64(out), f64(lse), 0.2)


@pytest.mark.parametrize("kind", ["peaked", "tiny", "huge", "zero", "mixed", "far"])
def test_attention_ranges(gpu_lib, kind):
    """One token taking all the weight; value scales far from 1, zero, or of very different sizes, where the largest weight
    is not the largest p; scores far from 0."""
    s = Setup(33, 1, 4, 1, 128, 64, [700])
    blocks = s.pages.reshape(-1, c.block_bytes(128))
    vs = blocks[:, 34 * 128:].copy().view(np.float32)
    q = s.rows(3, 4)
    if kind == "peaked":
        q *= 60
        q = c.to_bf16(q)
    if kind == "tiny":
        vs[:] *= 2.0 ** -70
    if kind == "huge":
        vs[:] *= 2.0 ** 90
    if kind == "zero":
        vs[:] = 0
    if kind == "mixed":
        vs[:] *= np.exp2(s.rng.integers(-30, 30, vs.shape)).astype(np.float32)
        vs[s.rng.random(vs.shape) < 0.1] = 0
    if kind == "far":
        q = c.to_bf16(q * 400)
    blocks[:, 34 * 128:] = vs.view(np.uint8).reshape(len(blocks), -1)
    s.upload()
    out, lse = attend(s, q, [3], 0.088)
    check_attention(s, q, [3], f64(out), f64(lse), 0.088)


@pytest.mark.parametrize("d,page", [(128, 32), (64, 32), (128, 256)])
def test_attention_batch_of_one_long_sequence(gpu_lib, d, page):
    """Enough (sequence, head) pairs that a sequence is one chunk: a wave's blocks span more than 64 pages (of 32
    tokens), eight waves read them; the short sequences beside it."""
    lens = [4096 - 7, 1, 0, 31, 33, 64] + [5] * 26 + [3000]
    s = Setup(37, 1, 8, 8, d, page, lens, cols=4096 // page)
    s.table[32, 70 * 32 // page] = -1  # a missing page beyond the 64th
    s.upload()
    q = s.rows(len(lens), 8)
    out, lse = attend(s, q, [1] * len(lens), 0.1)
    check_attention(s, q, [1] * len(lens), f64(out), f64(lse), 0.1, only=[0, 1, 2, 3, 4, 5, 32], heads=[0, 7])


@pytest.mark.parametrize("d,page,T", [(64, 32, 9), (128, 32, 9), (128, 64, 17)])
def test_attention_many_prompts(gpu_lib, d, page, T):
    """Four tiles of rows and whole sequences (1024 workgroups and more), pages looked up beyond the 64th of a wave."""
    lens = [2500, 40, T, 3, 0, 6100] + [20] * 122
    new = [T, T, T, min(T, 5), 0, T - 1] + [1] * 122
    s = Setup(38, 1, 64, 8, d, page, lens)
    q = s.rows(sum(new), 64)
    out, lse = attend(s, q, new, 0.1, max_new=T)
    check_attention(s, q, new, f64(out), f64(lse), 0.1, only=[0, 1, 2, 3, 5, 127], heads=[2])


@pytest.mark.parametrize("R,T", [(1, 1), (8, 4), (8, 5)])
def test_attention_of_a_large_cache(gpu_lib, R, T):
    """A length bound by which the cache exceeds the chip's caches (streaming loads), with one to four tiles; short and
    longer sequences, whose chunks merge in both ways."""
    lens = [9000, 700, 17, 5000]
    s = Setup(39, 1, 2 * R, 2, 128, 64, lens, cols=1 << 14)
    new = [T, min(T, 2), T, 1]
    q = s.rows(sum(new), 2 * R)
    out, lse = attend(s, q, new, 0.1, max_len=1 << 20, max_new=T)
    check_attention(s, q, new, f64(out), f64(lse), 0.1, heads=[1])
    # fewer chunks, by the bound: the same result within the tolerance
    out, lse = attend(s, q, new, 0.1, max_len=9000, max_new=T)
    check_attention(s, q, new, f64(out), f64(lse), 0.1, heads=[1])


def test_attention_scales_far_apart(gpu_lib):
    """Key scales of very different sizes within a block and from block to block, zero keys, queries near the ends of
    the range: the key factors' common power of two moves."""
    s = Setup(40, 1, 4, 1, 128, 64, [640, 95])
    blocks = s.pages.reshape(-1, c.block_bytes(128))
    ks = s.rng.uniform(0.1, 0.5, (len(blocks), 32, 4))
    for i in range(len(blocks)):  # a block's keys all of one power, a few of them zero
        ks[i] *= 2.0 ** s.rng.integers(-12, 13)
        ks[i][s.rng.random((32, 4)) < 0.1] *= 2.0 ** -6
        ks[i][s.rng.random((32, 4)) < 0.1] *= 2.0 ** -15
        if i % 4 == 1:
            ks[i] = 0.0
    blocks[:, 32 * 128:34 * 128] = c.bf16_bits(ks.reshape(len(blocks), 128)).view(np.uint8).reshape(len(blocks), -1)
    s.upload()
    for power in (-100, -20, 0, 4, 100):
        q = c.to_bf16(s.rows(3, 4) * 2.0 ** power)
        scale = float(np.float32(0.05 * 2.0 ** -min(power, 110)))
        out, lse = attend(s, q, [2, 1], scale)
        check_attention(s, q, [2, 1], f64(out), f64(lse), scale)


def test_attention_of_large_rows_at_right_angles(gpu_lib):
    """Queries and keys whose largest channels' product is beyond fp32, in different channels: every score is 0."""
    s = Setup(41, 1, 4, 1, 128, 64, [100])
    blocks = s.pages.reshape(-1, c.block_bytes(128))
    blocks[:, :16 * 128].reshape(-1, 32, 16, 4)[:, :, 0::4] = 0x88  # channels 0..31 of the keys: zeros
    ks = c.bf16_bits(np.full((len(blocks), 128), 2.0 ** 120)).view(np.uint8)
    blocks[:, 32 * 128:34 * 128] = ks.reshape(len(blocks), -1)
    s.upload()
    q = s.rows(2, 4) * 2.0 ** 120
    q[..., 32:] = 0
    q = c.to_bf16(q)
    out, lse = attend(s, q, [2], 1.0)
    check_attention(s, q, [2], f64(out), f64(lse), 1.0)


def test_attention_strides(gpu_lib):
    """Queries inside a fused projection's rows, head-major queries and outputs, and an output between guards."""
    s = Setup(34, 1, 8, 2, 64, 32, [90, 41])
    new, scale = [3, 2], 0.125
    q = s.rows(5, 8)
    want, wl = attend(s, q, new, scale)
    fused = torch.randn((5, 14, 64), device="cuda").to(torch.bfloat16)
    fused[:, 2:10] = bf16(q[0]).cuda()
    guarded = torch.full((5, 11, 72), -7.0, dtype=torch.bfloat16, device="cuda")
    step = B.Step(5, 3, torch.tensor([0, 3, 5], dtype=torch.int32, device="cuda"))
    B.tp_cache_attention(s.dims, s.cache, step, fused[:, 2:10], scale, 96, guarded[:, 1:9, :64])
    assert torch.equal(guarded[:, 1:9, :64], want[0])
    guarded[:, 1:9, :64] = -7.0
    assert bool((guarded == -7).all())
    heads = bf16(q[0]).cuda().transpose(0, 1).contiguous()  # [Hq][total][d]
    out = torch.empty_like(heads)
    B.tp_cache_attention(s.dims, s.cache, step, heads.transpose(0, 1), scale, 96, out.transpose(0, 1), wl)
    assert torch.equal(out.transpose(0, 1), want[0])
    # one query for all tokens and heads (broadcast: strides 0)
    one = bf16(q[0, :1, :1]).cuda()
    out = torch.empty((5, 8, 64), dtype=torch.bfloat16, device="cuda")
    B.tp_cache_attention(s.dims, s.cache, step, one.expand(5, 8, 64), scale, 96, out)
    same, _ = attend(s, np.broadcast_to(q[:, :1, :1], q.shape).copy(), new, scale)
    assert torch.equal(out, same[0])


@pytest.mark.parametrize("lens,new", [([90, 41], [3, 2]), ([9000, 70], [17, 1]), ([300], [100]), ([2000, 0], [1, 1])])
def test_attention_in_place(gpu_lib, lens, new):
    """Outputs on the queries' memory, with one to four tiles of rows, whole and in chunks."""
    s = Setup(42, 1, 8, 2, 128, 64, lens)
    q = s.rows(sum(new), 8)
    want, wl = attend(s, q, new, 0.1, max_len=max(lens))
    rows, lse = bf16(q).cuda(), torch.empty_like(wl)
    step = B.Step(sum(new), max(new), torch.from_numpy(offsets_of(new)).cuda())
    B.tp_cache_attention(s.dims, s.cache, step, rows, 0.1, max(lens), rows, lse)
    assert torch.equal(rows, want) and torch.equal(lse, wl)


def test_one_token_without_offsets_and_padded_batch(gpu_lib):
    """offsets = NULL: row b is sequence b's token; padded sequences have length 0, rows behind the batch stay."""
    s = Setup(35, 1, 8, 2, 128, 64, [100, 0, 33, 0], cols=2)
    q = s.rows(6, 8)
    out = torch.full((6, 8, 128), -7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((8, 6), -7.0, device="cuda")
    B.tp_cache_attention(s.dims, s.cache, B.Step(6), bf16(q[0]).cuda(), 0.1, 128, out, lse)
    torch.cuda.synchronize()
    check_attention(s, q, [1, 1, 1, 1], f64(out)[None], f64(lse)[None], 0.1)
    assert bool((out[4:] == -7).all()) and bool((lse[:, 4:] == -7).all())
    k, v = s.rows(6, 2), s.rows(6, 2)
    B.tp_cache_append(s.dims, s.cache, B.Step(6), bf16(k[0]).cuda(), bf16(v[0]).cuda())
    for b in (0, 2):
        for h in range(2):
            s.write(b, s.lens_[b] - 1, 0, h, c.quantise_key(k[0, b, h]), c.quantise_value(v[0, b, h]))
    s.check_pages()


def test_pool_beyond_4_gib(gpu_lib):
    """Pages whose offset passes 32 bits."""
    d, page, Hkv = 128, 256, 8
    dims = B.dims(1, 8, Hkv, d)
    each = B.tp_cache_page_bytes(dims, page) * Hkv
    num = (1 << 32) // each + 40
    small = Setup(36, 1, 8, Hkv, d, page, [600, 20])
    pool = torch.zeros(num * each, dtype=torch.uint8, device="cuda").view(num, Hkv, page // 32, -1)
    at = torch.arange(num - small.num, num, device="cuda")
    pool[at] = small.dev[0]
    table = torch.where(small.dtable >= 0, small.dtable + (num - small.num), -1).to(torch.int32)
    big = B.Cache(dims, pool, table, small.lens, page)
    q, k, v = (bf16(small.rows(2, 8)[0]).cuda() for _ in range(3))
    outs = []
    for cache in (small.cache, big):
        B.tp_cache_append(dims, cache, B.Step(2), k, v)
        out = torch.empty((2, 8, d), dtype=torch.bfloat16, device="cuda")
        B.tp_cache_attention(dims, cache, B.Step(2), q, 0.1, 768, out)
        kk = torch.empty((1, Hkv, 620, d), dtype=torch.bfloat16, device="cuda")
        vv = torch.empty_like(kk)
        B.tp_cache_read(dims, cache, B.Batch([0, 600, 620]), kk, vv)
        outs.append((out, kk, vv))
    assert all(torch.equal(a, b) for a, b in zip(*outs))
    assert torch.equal(pool[at], small.dev[0]) and not bool(pool[:num - small.num].any())


# ------------------------------------------------------------------------------ together
def test_evict_load_decode_read_evict(gpu_lib):
    """The way it is used: an eviction's compact cache into pages, decode steps, the answer read back and
    evicted again with the kept tokens."""
    L, Hq, Hkv, d, lens, budget, steps = 2, 8, 2, 64, [300, 150], 64, 5
    rng = np.random.default_rng(41)
    dims = B.dims(L, Hq, Hkv, d)
    n, scale = sum(lens), 0.125
    k, v = (bf16(rng.normal(size=(L, Hkv, n, d))).cuda() for _ in range(2))
    qg = bf16(rng.normal(size=(L, Hq, 16, d))).cuda()
    batch = B.Batch([0, 300, 450], [0, 8, 16])
    kw = dict(softmax_scale=scale, pool_k=5, qfmt=B.TP_QFMT_INT, bits=4, keep_budget=budget)
    bufs = B.evict_fused(dims, batch, qg, k, v, **kw)
    s = Setup(42, L, Hq, Hkv, d, 32, [budget + steps] * 2)
    kept = bufs.kept_offsets
    B.tp_cache_load(dims, s.cache, kept, bufs.k_c, bufs.v_q_c, bufs.scales_c, 4)
    kc = f64(bufs.k_c).reshape(L, Hkv, kept[-1], d)
    codes = bufs.v_q_c.cpu().numpy().reshape(L, Hkv, kept[-1], d // 2)
    vc = np.stack([codes & 15, codes >> 4], -1).reshape(L, Hkv, kept[-1], d).astype(int)
    vc = np.where(vc > 7, vc - 16, vc)
    sc = bufs.scales_c.cpu().numpy().reshape(L, Hkv, kept[-1])
    for b in range(2):
        for t in range(budget):
            for l in range(L):
                for h in range(Hkv):
                    i = kept[b] + t
                    s.write(b, t, l, h, c.quantise_key(kc[l, h, i]), (vc[l, h, i], sc[l, h, i]))
    s.check_pages()
    cs = table_of(400, d)
    rope = B.Rope(torch.from_numpy(cs).cuda(), d)
    for i in range(steps):
        s.lens_ = [budget + i + 1] * 2
        s.lens.copy_(torch.tensor(s.lens_, dtype=torch.int32))
        pos = np.array([300 + i, 150 + i], dtype=np.int32)
        qn, kn, vn = s.rows(2, Hq), s.rows(2, Hkv), s.rows(2, Hkv)
        qr = bf16(qn).cuda()
        B.tp_cache_append(dims, s.cache, B.Step(2), bf16(kn).cuda(), bf16(vn).cuda(), torch.from_numpy(pos).cuda(), rope, qr, qr)
        out = torch.empty((L, 2, Hq, d), dtype=torch.bfloat16, device="cuda")
        lse = torch.empty((L, Hq, 2), device="cuda")
        B.tp_cache_attention(dims, s.cache, B.Step(2), qr, scale, budget + steps, out, lse)
        for b in range(2):
            for l in range(L):
                for h in range(Hkv):
                    s.write(b, budget + i, l, h, c.quantise_key(c.rotate(kn[l, b, h], cs[pos[b]], d, 0)), c.quantise_value(vn[l, b, h]))
        s.check_pages()
        want = np.array([[[c.rotate(qn[l, b, h], cs[pos[b]], d, 0) for h in range(Hq)] for b in range(2)] for l in range(L)])
        same(f64(qr), want)
        check_attention(s, want, [1, 1], f64(out), f64(lse), scale)
    m = budget + steps
    k2 = torch.empty((L, Hkv, 2 * m, d), dtype=torch.bfloat16, device="cuda")
    v2 = torch.empty_like(k2)
    back = B.Batch([0, m, 2 * m], [0, 8, 16])
    B.tp_cache_read(dims, s.cache, back, k2, v2)
    for b in range(2):
        kk, vv, _ = c.held(s.pages, d, s.table[b], 32, 1, 0, m)
        same(f64(k2[1, 0, b * m:(b + 1) * m]), c.by_fp32(kk))
    kw["keep_budget"] = 20
    again = B.evict_fused(dims, back, qg, k2, v2, **kw)
    idx = again.kept_idx.view(L, Hkv, 40).cpu().numpy()
    assert np.all(np.diff(idx[..., :20]) > 0) and idx.min() >= 0 and idx.max() < m
    # the rows read back quantise to the codes that were held, so what is kept of them is held unchanged
    B.tp_cache_load(dims, s.cache, again.kept_offsets, again.k_c, again.v_q_c, again.scales_c, 4)
    s.lens.fill_(20)
    k3 = torch.empty((L, Hkv, 40, d), dtype=torch.bfloat16, device="cuda")
    v3 = torch.empty_like(k3)
    B.tp_cache_read(dims, s.cache, B.Batch([0, 20, 40]), k3, v3)
    assert torch.allclose(k3.float(), again.k_c.view_as(k3).float(), rtol=0, atol=0.51 * float(k2.abs().max()) / 7 * 1.01)


def test_captured_steps_with_shared_workspace(gpu_lib):
    """Two captured decode steps of different sequences on one workspace, replayed with lengths, positions and tokens
    changed in place, against eager calls; the program's own work between the replays."""
    setups = [Setup(51 + i, 1, 8, 2, 128, 64, [900, 1, 300], cols=16, spare=40) for i in range(2)]
    for s in setups:  # pages for growth
        free = [p for p in range(s.num) if p not in s.table]
        for b in range(3):
            for i in range(s.table.shape[1]):
                if s.table[b, i] < 0 and free:
                    s.table[b, i] = free.pop()
        s.upload()
    dims, step = setups[0].dims, B.Step(3)
    rope = B.Rope(torch.from_numpy(table_of(3000, 128)).cuda(), 128)
    ws = torch.empty(B.tp_cache_workspace_size(dims, setups[0].cache, step, 1024), dtype=torch.uint8, device="cuda")
    io = []
    for s in setups:
        t = {n: torch.zeros((3, h, 128), dtype=torch.bfloat16, device="cuda") for n, h in (("q", 8), ("k", 2), ("v", 2), ("qr", 8), ("o", 8))}
        t["pos"], t["lse"] = torch.zeros(3, dtype=torch.int32, device="cuda"), torch.zeros((8, 3), device="cuda")
        io.append(t)

    def call(s, t, cache):
        B.tp_cache_append(dims, cache, step, t["k"], t["v"], t["pos"], rope, t["q"], t["qr"])
        B.tp_cache_attention(dims, cache, step, t["qr"], 0.1, 1024, t["o"], t["lse"], ws)

    side = torch.cuda.Stream()
    graphs = []
    for s, t in zip(setups, io):
        with torch.cuda.stream(side):
            call(s, t, s.cache)
        side.synchronize()
        s.dev.copy_(torch.from_numpy(s.pages))
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            call(s, t, s.cache)
        graphs.append(g)
    rng = np.random.default_rng(53)
    for i in range(4):
        for s, t, g in zip(setups, io, graphs):
            s.lens.add_(1)
            for n in ("q", "k", "v"):
                t[n].copy_(bf16(rng.normal(size=t[n].shape)))
            t["pos"].copy_(torch.from_numpy(rng.integers(0, 3000, 3).astype(np.int32)))
            copy = s.dev.clone()
            g.replay()
            torch.cuda.synchronize()
            got = [t[n].clone() for n in ("qr", "o", "lse")] + [s.dev.clone()]
            for n in ("qr", "o", "lse"):
                t[n].zero_()
            call(s, t, B.Cache(dims, copy, s.dtable, s.lens, 64))
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, [t["qr"], t["o"], t["lse"], copy])), i
            s.pages = copy.cpu().numpy()
            s.lens_ = s.lens.tolist()
            check_attention(s, f64(t["qr"])[None], [1, 1, 1], f64(t["o"])[None], f64(t["lse"])[None], 0.1)


def test_two_streams(gpu_lib):
    """Two calls at once on streams of their own read one cache, each with its workspace."""
    s = Setup(61, 1, 8, 2, 64, 32, [3000, 500])
    q = [s.rows(2, 8) for _ in range(2)]
    want = [attend(s, x, [1, 1], 0.125) for x in q]
    step, streams = B.Step(2), [torch.cuda.Stream() for _ in range(2)]
    dev = [bf16(x[0]).cuda() for x in q]
    outs = [torch.zeros((2, 8, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(10):
        for st, x, out in zip(streams, dev, outs):
            B.tp_cache_attention(s.dims, s.cache, step, x, 0.125, 3008, out, stream=st)
    torch.cuda.synchronize()
    for out, (w, _) in zip(outs, want):
        assert torch.equal(out, w[0])
