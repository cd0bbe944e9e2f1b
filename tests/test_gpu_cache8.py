"""The paged 8-bit cache through the C ABI on the GPU, against the float64 oracle.

What is written is compared byte for byte over the whole pool, so what a call must leave alone is checked too.  The
attention's tolerances are those of cache_cases.py, which go by the keys and values held: a score is d exact products of
a code and a query, summed in fp32, times one factor; a weight times its value's scale is rounded to fp16."""
import math

import numpy as np
import pytest
import torch

import cache_cases as cc
import test_gpu_cache as T
from oracle import cache8_oracle as c
from oracle import cache_oracle as c4
from oracle import taskpress_oracle as o
from paper_2608_03276_amd import binding as B

pytestmark = pytest.mark.gpu
FMTS = [B.TP_QFMT_INT, B.TP_QFMT_FP8_E4M3]
bf16, f64, same, offsets_of, table_of = T.bf16, T.f64, T.same, T.offsets_of, T.table_of
by_fmt = pytest.mark.parametrize("fmt", FMTS, ids=["int", "fp8"])


class Setup(T.Setup):
    """A cache of random codes and ordinary scales with shuffled pages, on the host and on the GPU."""

    def __init__(self, seed, fmt, L, Hq, Hkv, d, page, lens, cols=None, spare=2):
        self.rng = np.random.default_rng(seed)
        self.fmt, self.L, self.Hq, self.Hkv, self.d, self.page, self.lens_ = fmt, L, Hq, Hkv, d, page, list(lens)
        self.dims = B.dims(L, Hq, Hkv, d)
        need = [-(-max(n, 0) // page) for n in lens]
        self.num = sum(need) + spare
        order = self.rng.permutation(self.num)
        self.table = np.full((len(lens), cols or max(max(need), 1)), -1, dtype=np.int32)
        i = 0
        for b, n in enumerate(need):
            self.table[b, :n] = order[i:i + n]
            i += n
        size = c.block_bytes(d)
        self.pages = self.rng.integers(1, 256, (L, self.num, Hkv, page // 32, size)).astype(np.uint8)
        if fmt == c.FP8:
            self.pages[(self.pages & 0x7F) == 0x7F] = 0x30
        blocks = self.blocks()
        # scores and values of order 1: codes have a root mean square of 73 (integers), 145 (e4m3)
        vs = self.rng.uniform(0.1, 0.5, (len(blocks), 32)) / 20 * np.where(self.rng.random((len(blocks), 32)) < 0.05, 20, 1)
        self.set_value_scales(vs)
        self.set_key_scales(self.rng.uniform(0.1, 0.5, len(blocks)) / 40)
        self.upload()

    def blocks(self):
        return self.pages.reshape(-1, c.block_bytes(self.d))

    def set_value_scales(self, x):
        self.blocks()[:, 64 * self.d:64 * self.d + 128] = np.ascontiguousarray(x, dtype=np.float32).view(np.uint8)

    def set_key_scales(self, x):
        self.blocks()[:, 64 * self.d + 128:64 * self.d + 132] = np.ascontiguousarray(x, dtype=np.float32)[:, None].view(np.uint8)

    def upload(self):
        self.dev = torch.from_numpy(self.pages.copy()).cuda()
        self.lens = torch.tensor(self.lens_, dtype=torch.int32, device="cuda")
        self.dtable = torch.from_numpy(self.table.copy()).cuda()
        self.cache = B.Cache8(self.dims, self.dev, self.dtable, self.lens, self.page, self.fmt)

    def write(self, b, start, layer, head, keys, values):
        """One call's tokens of a sequence: its first token, {token: key row}, {token: (bytes, scale)}."""
        for j in sorted({t // 32 for t in keys}):
            at = c4.place_of(self.table[b], self.num, self.page, 32 * j)
            if at is None:
                continue
            block = self.pages[layer, at[0], head, at[1]]
            mine = [t for t in keys if t // 32 == j]
            c.write_keys(block, self.d, self.fmt, max(start - 32 * j, 0), {t % 32: keys[t] for t in mine})
            for t in mine:
                c.write_value(block, self.d, t % 32, *values[t])

    def check_pages(self):
        got = self.dev.cpu().numpy()
        if not np.array_equal(got, self.pages):
            bad = np.argwhere(got != self.pages)
            raise AssertionError(f"{len(bad)} bytes differ, first at {bad[0]}: {got[tuple(bad[0])]}, expected "
                                 f"{self.pages[tuple(bad[0])]} (block bytes {c.block_bytes(self.d)})")

    def held(self, b, layer, head, n):
        return c.held(self.pages, self.d, self.fmt, self.table[b], self.page, layer, head, n)


def append_expected(s, lens, new, off, k, v, q, cs, pos, r, style, most=None, cap=None):
    """Writes what an append writes into the setup's pages and returns the query rows expected (-7: left alone)."""
    want = np.full(q.shape, -7.0)
    for b in range(len(lens)):
        n = lens[b] if cap is None or 0 <= lens[b] <= cap else 0
        if most is not None and new[b] > most:
            continue
        good = [t for t in range(new[b]) if cs is None or 0 <= pos[off[b] + t] < len(cs)]
        turn = (lambda x, row: c4.rotate(x, cs[pos[row]], r, style)) if cs is not None else (lambda x, row: x)
        for l in range(s.L):
            for t in good:
                for h in range(s.Hq):
                    want[l, off[b] + t, h] = turn(q[l, off[b] + t, h], off[b] + t)
            for h in range(s.Hkv):
                there = [t for t in good if n - new[b] + t >= 0 and n > 0]
                keys = {n - new[b] + t: turn(k[l, off[b] + t, h], off[b] + t) for t in there}
                vals = {n - new[b] + t: c.quantise_value(v[l, off[b] + t, h], s.fmt) for t in there}
                s.write(b, max(n - new[b], 0), l, h, keys, vals)
    return want


# ------------------------------------------------------------------------------ append
@by_fmt
@pytest.mark.parametrize("case", T.APPENDS, ids=[f"L{a[0]}h{a[1]}-{a[2]}d{a[3]}p{a[4]}r{a[7]}s{a[8]}" for a in T.APPENDS])
def test_append(gpu_lib, case, fmt):
    L, Hq, Hkv, d, page, lens, new, r, style, with_q = case
    s = Setup(11, fmt, L, Hq, Hkv, d, page, lens)
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
    B.tp_cache8_append(s.dims, s.cache, step, bf16(k).cuda(), bf16(v).cuda(), **kw)
    torch.cuda.synchronize()
    want = append_expected(s, lens, new, off, k, v, q, cs, pos, r, style)
    s.check_pages()
    same(f64(q_out), want if with_q else np.full(q.shape, -7.0))


@by_fmt
@pytest.mark.parametrize("style", [0, 1])
@pytest.mark.parametrize("Hq,Hkv,new", [(33, 3, [1, 1]), (32, 8, [5, 2]), (33, 3, [3, 1]), (48, 8, [2, 33]), (72, 8, [40, 1]), (130, 2, [4, 2])])
def test_append_many_query_heads(gpu_lib, Hq, Hkv, new, style, fmt):
    """Query rows of one to nine passes of a workgroup, whole and not, written apart and in place."""
    lens = [n + 30 for n in new]
    s = Setup(17, fmt, 1, Hq, Hkv, 128, 32, lens)
    off, total = offsets_of(new), sum(new) + 1
    k, v, q = (s.rows(total, h) for h in (Hkv, Hkv, Hq))
    cs = table_of(200, 96)
    pos = s.rng.integers(0, 200, total).astype(np.int32)
    pos[1] = -1 if sum(new) > 2 else pos[1]
    q_out = torch.full(q.shape, -7.0, dtype=torch.bfloat16, device="cuda")
    step = B.Step(total, max(new), torch.from_numpy(off).cuda())
    kw = dict(positions=torch.from_numpy(pos).cuda(), rope=B.Rope(torch.from_numpy(cs).cuda(), 96, style))
    q_dev = bf16(q).cuda()
    B.tp_cache8_append(s.dims, s.cache, step, bf16(k).cuda(), bf16(v).cuda(), q=q_dev, q_out=q_out, **kw)
    want = append_expected(s, lens, new, off, k, v, q, cs, pos, 96, style)
    s.check_pages()
    same(f64(q_out), want)
    s.upload()
    B.tp_cache8_append(s.dims, s.cache, step, bf16(k).cuda(), bf16(v).cuda(), q=q_dev, q_out=q_dev, **kw)
    same(f64(q_dev), np.where(want == -7.0, q, want))


@by_fmt
@pytest.mark.parametrize("d,page", [(64, 32), (128, 64)])
def test_append_raises_scales(gpu_lib, d, page, fmt):
    """Token by token through two blocks, with keys of growing, falling, zero and equal size: the scale rises by powers of
    two, the held codes are rounded again, and nothing else changes."""
    sizes = [0.0, 0.0, 1.0, 1.0, 0.5, 1.01, 2.0, 2.03125, 3.0, 0.0, 100.0, 1e-3, 1600.0, 1610.0, 5.0, 2.0 ** 20, 1.0] + [2.0 ** 21] * 8 \
        + [2.0 ** 22 * 1.5 ** i for i in range(9)] + [1e-30, 1e30, 1e31, 2e31]
    s = Setup(16, fmt, 1, 2, 2, d, page, [64], cols=2)
    for t, size in enumerate(sizes):
        s.lens_ = [t + 1]
        s.lens.fill_(t + 1)
        k = s.rows(1, 2)
        k[0, 0] = c4.to_bf16(k[0, 0] / np.abs(k[0, 0]).max(1, keepdims=True) * size)  # both heads' largest is `size`
        v = s.rows(1, 2)
        B.tp_cache8_append(s.dims, s.cache, B.Step(1), bf16(k[0]).cuda(), bf16(v[0]).cuda())
        append_expected(s, [t + 1], [1], [0, 1], k, v, np.zeros((1, 1, 2, d)), None, None, 0, 0)
        s.check_pages()
    # several at once into a block that holds some, the largest the last
    s.lens_ = [len(sizes) + 9]
    s.lens.fill_(s.lens_[0])
    k, v = s.rows(9, 2) * 2.0 ** 100, s.rows(9, 2)
    k[0, 8] *= 7
    k = c4.to_bf16(k)
    B.tp_cache8_append(s.dims, s.cache, B.Step(9, 9, torch.tensor([0, 9], dtype=torch.int32, device="cuda")), bf16(k[0]).cuda(),
                       bf16(v[0]).cuda())
    append_expected(s, s.lens_, [9], [0, 9], k, v, np.zeros((1, 9, 2, d)), None, None, 0, 0)
    s.check_pages()
    # cut back and appended again: the last block keeps its scale
    s.lens_ = [len(sizes) + 2]
    s.lens.fill_(s.lens_[0])
    k, v = s.rows(1, 2), s.rows(1, 2)
    B.tp_cache8_append(s.dims, s.cache, B.Step(1), bf16(k[0]).cuda(), bf16(v[0]).cuda())
    append_expected(s, s.lens_, [1], [0, 1], k, v, np.zeros((1, 1, 2, d)), None, None, 0, 0)
    s.check_pages()


@by_fmt
@pytest.mark.parametrize("d,new", [(64, 1), (128, 1), (128, 3), (64, 40)])
def test_append_beside_scales_of_any_kind(gpu_lib, d, new, fmt):
    """Blocks with earlier tokens and a scale that is none (0, negative, NaN, infinite): the keys get one of their own.  A
    positive finite one, whoever left it, is the block's, however large or small."""
    none, some = [0.0, -0.0, -1.0, -1e30, math.nan, -math.nan, math.inf, -math.inf], [1e-30, 1e-42, 0.01, 1e30, 3e38]
    held = np.array(none + some, dtype=np.float32)
    s = Setup(18, fmt, 1, 2, 2, d, 64, [5 + new] * len(held))
    for b, x in enumerate(held):
        at = c4.place_of(s.table[b], s.num, s.page, 0)
        s.pages[0, at[0], :, at[1], 64 * d + 128:64 * d + 132] = np.array([x]).view(np.uint8)
    s.upload()
    off, total = offsets_of([new] * len(held)), new * len(held)
    k, v = s.rows(total, 2), s.rows(total, 2)
    B.tp_cache8_append(s.dims, s.cache, B.Step(total, new, torch.from_numpy(off).cuda()), bf16(k).cuda(), bf16(v).cuda())
    append_expected(s, s.lens_, [new] * len(held), off, k, v, np.zeros((1, total, 2, d)), None, None, 0, 0)
    s.check_pages()
    first = min(new, 27)  # the new tokens in the sequences' first blocks
    for b in range(len(none)):
        for h in range(2):
            rows = k[0, off[b]:off[b] + first, h]
            scale, got = np.float32(np.abs(rows).max() / c.qmax(fmt)), s.held(b, 0, h, 5 + first)[0][5:]
            # half a step, or half of e4m3's last place of a normal or subnormal code; 2^-24 each for scale and quotient
            most = scale / 2 if fmt == c.INT else np.maximum(np.abs(rows) * 2.0 ** -4, scale * 2.0 ** -10)
            assert np.all(np.abs(got - rows) <= most + np.abs(rows) * 2.0 ** -23), (b, h)


@by_fmt
@pytest.mark.parametrize("power", [-141, -133, -126, -110, -70, -60, 0, 60, 100, 120])
@pytest.mark.parametrize("d", [64, 128])
def test_append_odd_values(gpu_lib, d, power, fmt):
    """Keys and values at the edges of the format: every code's border, the smallest and largest numbers, in blocks of
    any size and beside a token that was held."""
    s = Setup(12, fmt, 1, 2, 2, d, 32, [33, 65])
    Q = c.qmax(fmt)
    k, v = s.rows(97, 2), s.rows(97, 2)
    codes = np.arange(127) + 0.5 if fmt == c.INT else (c.codes_of(np.arange(126, dtype=np.uint8), fmt) + c.codes_of(np.arange(1, 127, dtype=np.uint8), fmt)) / 2
    for t in range(97):
        m = 1 + s.rng.integers(0, 128, (2, 1)) / 128 if t % 3 else np.full((2, 1), Q / 2.0 ** 8)
        for x in (k, v):
            x[0, t] = m * s.rng.choice(codes, (2, d)) / Q * s.rng.choice([-1, 1], (2, d)) * (1 + s.rng.choice([-1, 0, 1], (2, d)) * 2.0 ** -8)
            x[0, t, :, 0] = m[:, 0]
    k[0, 5] = v[0, 5] = 0
    k[0, 6], v[0, 6] = -0.0, -0.0
    k, v = (c4.to_bf16(x * 2.0 ** power) for x in (k, v))
    if power == 120:
        k[0, 40] = v[0, 40] = c4._MAX_BF16
        k[0, 41] = v[0, 41] = -c4._MAX_BF16
    off = np.array([0, 33, 97], dtype=np.int32)
    s.lens_ = [33, 65]
    step = B.Step(97, 64, torch.from_numpy(off).cuda())
    s.set_key_scales(np.full(len(s.blocks()), 2.0 ** (power - 9) * 1.2345))
    s.upload()
    B.tp_cache8_append(s.dims, s.cache, step, bf16(k).cuda(), bf16(v).cuda())
    append_expected(s, s.lens_, [33, 64], off, k, v, np.zeros((1, 97, 2, d)), None, None, 0, 0)
    s.check_pages()


@by_fmt
def test_append_leaves_out_what_is_out_of_range(gpu_lib, fmt):
    """Lengths, offsets, pages and positions that no token has: nothing is written for them."""
    new = [2, 2, 3, 2, 2, 2, 5]
    lens = [40, 41, 2, 64, 1000, -5, 64]  # 2 < 3 new: the first is before the start; 1000 and -5 count as 0
    s = Setup(14, fmt, 1, 4, 2, 64, 32, [min(max(n, 0), 64) for n in lens], cols=2)
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
    B.tp_cache8_append(s.dims, s.cache, step, bf16(k).cuda(), bf16(v).cuda(), torch.from_numpy(pos).cuda(),
                       B.Rope(torch.from_numpy(cs).cuda(), 64), bf16(q[0]).cuda(), q_out)
    want = append_expected(s, lens, new, off, k, v, q, cs, pos, 64, 0, most=3, cap=64)
    s.check_pages()
    same(f64(q_out), want[0])


@by_fmt
@pytest.mark.parametrize("bad", [[0, 3, 2, 5], [0, 2, 9, 5], [-1, 2, 4, 5], [3, 4, 5, 6]])
def test_append_bad_offsets(gpu_lib, bad, fmt):
    """Ranges that decrease or leave the tensors count as empty; the others are written."""
    s = Setup(15, fmt, 1, 2, 1, 64, 32, [30, 31, 32])
    k, v = s.rows(5, 1), s.rows(5, 1)
    B.tp_cache8_append(s.dims, s.cache, B.Step(5, 4, torch.tensor(bad, dtype=torch.int32, device="cuda")), bf16(k).cuda(),
                       bf16(v).cuda())
    good = [bad[b + 1] - bad[b] if 0 <= bad[b] < bad[b + 1] <= 5 else 0 for b in range(3)]
    append_expected(s, [n if g else 0 for n, g in zip(s.lens_, good)], good, bad, k, v, np.zeros((1, 5, 2, 64)), None, None, 0, 0)
    s.check_pages()


# ------------------------------------------------------------------------------ load and read
@pytest.mark.parametrize("fmt,bits", [(B.TP_QFMT_INT, 2), (B.TP_QFMT_INT, 4), (B.TP_QFMT_INT, 5), (B.TP_QFMT_INT, 8),
                                      (B.TP_QFMT_FP8_E4M3, 0)])
@pytest.mark.parametrize("L,Hkv,d,page,kept", [(2, 2, 64, 32, [70, 0, 32, 1]), (1, 3, 128, 128, [129, 31]), (3, 1, 128, 64, [5])])
def test_load(gpu_lib, fmt, bits, L, Hkv, d, page, kept):
    s = Setup(21, fmt, L, Hkv, Hkv, d, page, kept)
    if len(kept) > 3:
        s.table[0, 1] = -1  # tokens 32..63 have no page
        s.upload()
    n = sum(kept)
    k = c4.to_bf16(s.rng.normal(size=(L, Hkv, n, d)))
    v = bf16(s.rng.standard_t(3, size=(L, Hkv, n, d))).cuda()
    scales = torch.empty((L, Hkv, n), device="cuda")
    row = B.row_bytes(fmt, bits, d)
    v_q = torch.empty((L, Hkv, n, row), dtype=torch.uint8, device="cuda")
    B.tp_quantize_v_scales(s.dims, B.Batch([0, n]), v, fmt, bits, scales, v_q)
    off = offsets_of(kept).tolist()
    B.tp_cache8_load(s.dims, s.cache, off, bf16(k).cuda(), v_q, scales, bits)
    vv = f64(v)
    for b in range(len(kept)):
        for l in range(L):
            for h in range(Hkv):
                rows = vv[l, h, off[b]:off[b + 1]]
                if not len(rows):
                    continue
                g = o.value_scales(rows, fmt, bits)
                codes = o.quantize_values(rows, g, fmt, bits)
                codes = codes if fmt == c.FP8 else (codes.astype(int) + 128).astype(np.uint8)
                s.write(b, 0, l, h, {t: k[l, h, off[b] + t] for t in range(kept[b])}, {t: (codes[t], g[t]) for t in range(kept[b])})
    s.check_pages()


@by_fmt
@pytest.mark.parametrize("d,page", [(64, 32), (128, 64), (128, 256)])
def test_read(gpu_lib, d, page, fmt):
    lens = [300, 5, 64, 0, 128]
    s = Setup(22, fmt, 2, 2, 2, d, page, lens, spare=3)
    s.table[2, 0] = -3  # a sequence whose first page is missing
    s.lens_[4] = 90     # fewer tokens than its pages hold
    s.upload()
    first, count = [37, 0, 0, 0, 60], [263, 9, 64, 3, 68]
    off = offsets_of(count).tolist()
    k = torch.full((2, 2, off[-1], d), -7.0, dtype=torch.bfloat16, device="cuda")
    v = torch.full_like(k, -7.0)
    B.tp_cache8_read(s.dims, s.cache, B.Batch(off), k, v, first)
    for b in range(5):
        for l in range(2):
            for h in range(2):
                kk, vv, _ = s.held(b, l, h, s.lens_[b])
                want = np.zeros((2, count[b], d))
                m = max(0, min(s.lens_[b] - first[b], count[b]))
                want[0, :m], want[1, :m] = kk[first[b]:first[b] + m], vv[first[b]:first[b] + m]
                want = c4.by_fp32(want)
                same(f64(k[l, h, off[b]:off[b + 1]]), want[0])
                same(f64(v[l, h, off[b]:off[b + 1]]), want[1])
    B.tp_cache8_read(s.dims, s.cache, B.Batch(off), k, v)  # from the start
    kk, vv, _ = s.held(0, 1, 1, 263)
    same(f64(k[1, 1, :263]), c4.by_fp32(kk))
    same(f64(v[1, 1, :263]), c4.by_fp32(vv))


@by_fmt
@pytest.mark.parametrize("d", [64, 128])
def test_read_more_than_the_caches_hold(gpu_lib, d, fmt):
    """Outputs above 256 MB: the same rows, zeros behind the sequences."""
    s = Setup(23, fmt, 1, 8, 8, d, 64, [300, 97])
    few = torch.empty((8, 397, d), dtype=torch.bfloat16, device="cuda")
    fewv = torch.empty_like(few)
    B.tp_cache8_read(s.dims, s.cache, B.Batch([0, 297, 397]), few, fewv, [3, 0])
    n = (1 << 28) // (8 * d * 4) + 333
    k = torch.full((1, 8, n, d), -7.0, dtype=torch.bfloat16, device="cuda")
    v = torch.full_like(k, -7.0)
    B.tp_cache8_read(s.dims, s.cache, B.Batch([0, 297, n]), k, v, [3, 0])
    for got, want in ((k, few), (v, fewv)):
        assert torch.equal(got[0, :, :394], want[:, :394])
        assert not bool(got[0, :, 394:].any())


# ------------------------------------------------------------------------------ attention
def attend(s, q, new, scale, max_len=None, total=None, max_new=None, lse=True, stream=None, ws=None):
    off = offsets_of(new)
    total = total or q.shape[1]
    step = B.Step(total, max_new or max(max(new), 1), torch.from_numpy(off).cuda())
    out = torch.full((s.L, total, s.Hq, s.d), -7.0, dtype=torch.bfloat16, device="cuda")
    l = torch.full((s.L, s.Hq, total), -7.0, device="cuda") if lse else None
    B.tp_cache8_attention(s.dims, s.cache, step, bf16(q).cuda(), scale, max_len or s.table.shape[1] * s.page, out, l, ws, stream)
    torch.cuda.synchronize()
    return out, l


def check_attention(s, q, new, got_o, got_lse, scale, only=None, heads=None):
    """Every row (of the sequences in `only`, the KV heads in `heads`) within its bound."""
    off, R, cap = offsets_of(new), s.Hq // s.Hkv, s.table.shape[1] * s.page
    got_o, got_lse = f64(got_o), f64(got_lse)
    for b in range(len(new)) if only is None else only:
        n = s.lens_[b] if 0 <= s.lens_[b] <= cap else 0
        for l in range(s.L):
            for h in range(s.Hkv) if heads is None else heads:
                k, v, there = s.held(b, l, h, n)
                for t in range(new[b]):
                    visible = there & (np.arange(n) <= n - new[b] + t)
                    for hq in range(h * R, (h + 1) * R):
                        bound = cc.bounds(q[l, off[b] + t, hq], k, v, visible, scale)
                        go, gl = got_o[l, off[b] + t, hq], got_lse[l, hq, off[b] + t]
                        assert cc.accepts(go, gl, bound), ((b, l, hq, t), float(np.max(np.abs(go - bound[0]) / np.maximum(bound[2], 1e-300))),
                                                           gl, bound[1], bound[3])


@by_fmt
@pytest.mark.parametrize("case", T.ATTENDS, ids=[f"L{a[0]}h{a[1]}-{a[2]}d{a[3]}n{max(a[5])}t{max(a[6])}" for a in T.ATTENDS])
def test_attention(gpu_lib, case, fmt):
    L, Hq, Hkv, d, page, lens, new = case
    s = Setup(31, fmt, L, Hq, Hkv, d, page, lens)
    total = sum(new) + 1  # a row of no sequence
    q = s.rows(total, Hq, 1.5)
    out, lse = attend(s, q, new, 1 / math.sqrt(d))
    check_attention(s, q, new, out, lse, 1 / math.sqrt(d))
    assert bool((out[:, -1] == -7).all()) and bool((lse[:, :, -1] == -7).all())
    again, l2 = attend(s, q, new, 1 / math.sqrt(d))
    assert torch.equal(out, again) and torch.equal(lse, l2)
    alone, _ = attend(s, q, new, 1 / math.sqrt(d), lse=False)
    assert torch.equal(out, alone)


@by_fmt
@pytest.mark.parametrize("d", [64, 128])
def test_attention_ignores_what_is_not_held(gpu_lib, d, fmt):
    """NaN codes and NaN, infinite and negative scales in slots and pages beyond the sequences, missing pages, lengths that
    do not count."""
    lens = [37, 100, 64, 161, 50, 31]
    s = Setup(32, fmt, 1, 4, 2, d, 32, lens, cols=6)
    mine = set(s.table[s.table >= 0].tolist())
    kb, vb = c.places(d)
    for p in range(s.num):
        if p not in mine:
            s.pages[0, p] = 0xFF
    for b, n in enumerate(lens):
        if n % 32:
            at = c4.place_of(s.table[b], s.num, s.page, n - 1)
            for h in range(2):
                blk = s.pages[0, at[0], h, at[1]]
                blk[64 * d:64 * d + 128].view(np.float32)[n % 32:] = [np.nan, np.inf, -np.inf][(b + h) % 3]
                blk[kb[n % 32:]] = 0x7F
                blk[vb[n % 32:]] = [0x7F, 0xFF][h]
    s.table[1, 1] = -1          # tokens 32..63 of sequence 1
    s.table[2] = s.num + 5      # sequence 2 has no pages at all
    s.lens_[4] = 6 * 32 + 1     # beyond its pages: counts as empty
    s.pages[0, 0] = s.pages[0, 0] if 0 in s.table else 0xFF  # what a missing page's loads see
    s.upload()
    for new in ([2, 1, 1, 40, 1, 1], [1, 1, 1, 1, 1, 1], [30, 20, 17, 3, 1, 31]):
        q = s.rows(sum(new), 4)
        out, lse = attend(s, q, new, 0.2)
        check_attention(s, q, new, out, lse, 0.2)
    # a bound below a sequence's length empties that one only
    s.lens_[4] = 50
    s.upload()
    new = [2, 1, 1, 40, 1, 1]
    q = s.rows(sum(new), 4)
    out, lse = attend(s, q, new, 0.2, max_len=128)
    s.lens_[3] = 10 ** 9
    check_attention(s, q, new, out, lse, 0.2)


@by_fmt
@pytest.mark.parametrize("kind", ["peaked", "tiny", "huge", "zero", "mixed", "far", "keys", "none"])
def test_attention_ranges(gpu_lib, kind, fmt):
    """One token taking all the weight; value scales far from 1, zero, or of very different sizes; scores far from 0; key
    scales of very different sizes from block to block, zero blocks among them; keys that are all 0."""
    s = Setup(33, fmt, 1, 4, 1, 128, 64, [700])
    vs = s.blocks()[:, 64 * 128:64 * 128 + 128].copy().view(np.float32)
    ks = s.blocks()[:, 64 * 128 + 128:64 * 128 + 132].copy().view(np.float32)[:, 0]
    q = s.rows(3, 4)
    if kind == "peaked":
        q = c4.to_bf16(q * 60)
    if kind == "tiny":
        vs *= np.float32(2.0 ** -70)
    if kind == "huge":
        vs *= np.float32(2.0 ** 90)
    if kind == "zero":
        vs[:] = 0
    if kind == "mixed":
        vs *= np.exp2(s.rng.integers(-30, 30, vs.shape)).astype(np.float32)
        vs[s.rng.random(vs.shape) < 0.1] = 0
    if kind == "far":
        q = c4.to_bf16(q * 400)
    if kind == "keys":
        ks *= np.exp2(s.rng.integers(-40, 3, ks.shape)).astype(np.float32)
        ks[::5] = 0
    if kind == "none":
        ks[:] = 0
    s.set_value_scales(vs)
    s.set_key_scales(ks)
    s.upload()
    out, lse = attend(s, q, [3], 0.088)
    check_attention(s, q, [3], out, lse, 0.088)


@by_fmt
@pytest.mark.parametrize("new", [[2, 1], [20, 30]])
def test_attention_powers_that_cancel(gpu_lib, new, fmt):
    """Queries, keys and the scores' factor near the ends of fp32's range, with scores of order 1."""
    s = Setup(40, fmt, 1, 4, 1, 128, 64, [640, 95])
    base = s.rng.uniform(0.1, 0.5, len(s.blocks())) / 40
    for key, query, factor in ((0, 0, 0), (118, -120, 0), (-100, 100, 0), (-118, 0, 118), (100, 20, -120), (-110, -20, 120)):
        s.set_key_scales(base * 2.0 ** key)
        s.upload()
        q = c4.to_bf16(s.rows(sum(new), 4) * 2.0 ** query)
        scale = float(np.float32(0.05 * 2.0 ** (2 + factor if key == 118 else factor)))
        out, lse = attend(s, q, new, scale)
        check_attention(s, q, new, out, lse, scale)


@by_fmt
@pytest.mark.parametrize("n", [90, 9000])
@pytest.mark.parametrize("T_", [1, 6, 20])
@pytest.mark.parametrize("d", [64, 128])
def test_attention_scores_beyond_fp32(gpu_lib, d, T_, n, fmt):
    """A row with a score of +infinity or a query that is not finite has o and lse NaN; a score of -infinity is a key that
    is not seen.  The rows beside it keep their results."""
    s = Setup(72, fmt, 1, 4, 2, d, 64, [n])
    kb, _ = c.places(d)
    blocks = s.blocks()
    blocks[:, kb[:, :32].ravel()] = c.bytes_of([100.0], fmt)[0]  # channels 0..31: above 0
    blocks[:, kb[:, 32:].ravel()] = np.where(blocks[:, kb[:, 32:].ravel()] == 0, 1, blocks[:, kb[:, 32:].ravel()])
    s.upload()
    kinds = ["ordinary", "up", "down", "nan", "inf", "both"]
    q = s.rows(T_, 4)
    for t in range(T_):
        kind = kinds[(t + 1) % 6] if T_ > 1 else "up"
        if kind in ("up", "down", "both"):
            rows = slice(1, None, 2) if kind == "both" else slice(None)  # both: one row of two ordinary
            q[0, t, rows] = 0.0
            q[0, t, rows, :32] = -2.0 ** 60 if kind == "down" else 2.0 ** 60
    q = c4.to_bf16(q)
    finite = q.copy()
    for t in range(T_):
        kind = kinds[(t + 1) % 6] if T_ > 1 else "up"
        if kind in ("nan", "inf"):
            q[0, t, :, 40] = np.nan if kind == "nan" else -np.inf
    out, lse = attend(s, q, [T_], 0.1)
    out, lse = f64(out)[0], f64(lse)[0]
    held = [s.held(0, 0, h, n) for h in range(2)]
    for t in range(T_):
        kind = kinds[(t + 1) % 6] if T_ > 1 else "up"
        for h in range(4):
            tag, got, l = (kind, t, h), out[t, h], lse[h, t]
            if kind in ("up", "nan", "inf") or (kind == "both" and h % 2 == 1):
                assert np.isnan(l) and np.isnan(got).all(), (tag, l, got[:4])
            elif kind == "down":
                assert l == -math.inf and not got.any(), (tag, l)
            else:
                k, v, _ = held[h // 2]
                assert cc.accepts(got, l, cc.bounds(finite[0, t, h], k, v, np.arange(n) <= n - T_ + t, 0.1)), tag


def test_rows_that_see_nothing_beside_rows_that_are_not_finite(gpu_lib):
    """More new tokens than are held: rows before the start see nothing and are 0, whatever their queries."""
    s = Setup(73, c.FP8, 1, 4, 2, 64, 32, [5])
    q = s.rows(9, 4)
    q[0, 1] = np.nan
    q[0, 7] = np.inf
    out, lse = attend(s, q, [9], 0.1)
    out, lse = f64(out)[0], f64(lse)[0]
    assert not out[:4].any() and np.all(lse[:, :4] == -math.inf)
    assert np.isnan(out[7]).all() and np.isnan(lse[:, 7]).all()
    assert np.isfinite(out[[4, 5, 6, 8]]).all()


@by_fmt
@pytest.mark.parametrize("d,page", [(128, 32), (64, 32), (128, 256)])
def test_attention_batch_of_one_long_sequence(gpu_lib, d, page, fmt):
    """Enough (sequence, head) pairs that a sequence is one chunk: a wave's blocks span more than 64 pages (of 32
    tokens), eight waves read them; the short sequences beside it."""
    lens = [4096 - 7, 1, 0, 31, 33, 64] + [5] * 26 + [3000]
    s = Setup(37, fmt, 1, 8, 8, d, page, lens, cols=4096 // page)
    s.table[32, 70 * 32 // page] = -1  # a missing page beyond the 64th
    s.upload()
    q = s.rows(len(lens), 8)
    out, lse = attend(s, q, [1] * len(lens), 0.1)
    check_attention(s, q, [1] * len(lens), out, lse, 0.1, only=[0, 1, 2, 3, 4, 5, 32], heads=[0, 7])


@by_fmt
@pytest.mark.parametrize("d,page,T_", [(64, 32, 9), (128, 64, 17)])
def test_attention_many_prompts(gpu_lib, d, page, T_, fmt):
    """Four tiles of rows and whole sequences, pages looked up beyond the 64th of a wave."""
    lens = [2500, 40, T_, 3, 0, 6100] + [20] * 122
    new = [T_, T_, T_, min(T_, 5), 0, T_ - 1] + [1] * 122
    s = Setup(38, fmt, 1, 64, 8, d, page, lens)
    q = s.rows(sum(new), 64)
    out, lse = attend(s, q, new, 0.1, max_new=T_)
    check_attention(s, q, new, out, lse, 0.1, only=[0, 1, 2, 3, 5, 127], heads=[2])


@by_fmt
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("R,T_", [(1, 1), (8, 4), (8, 5)])
def test_attention_of_a_large_cache(gpu_lib, R, T_, d, fmt):
    """A length bound by which the cache exceeds the chip's caches (streaming loads), with one to four tiles; short and
    longer sequences, whose chunks merge in both ways."""
    lens = [9000, 700, 17, 5000]
    s = Setup(39, fmt, 1, 2 * R, 2, d, 64, lens, cols=1 << 14)
    new = [T_, min(T_, 2), T_, 1]
    q = s.rows(sum(new), 2 * R)
    out, lse = attend(s, q, new, 0.1, max_len=1 << 20, max_new=T_)
    check_attention(s, q, new, out, lse, 0.1, heads=[1])
    out, lse = attend(s, q, new, 0.1, max_len=9000, max_new=T_)  # fewer chunks, by the bound
    check_attention(s, q, new, out, lse, 0.1, heads=[1])


@by_fmt
@pytest.mark.parametrize("d,most", [(128, 4096), (128, 2048), (64, 4096)])
def test_attention_of_many_whole_sequences(gpu_lib, d, most, fmt):
    """Eight waves a sequence, streamed (496 pairs of up to 4096 tokens are 529 MB, at d = 64 269) and not."""
    lens = [2500, 4, 0, 700] + [1 + i % 40 for i in range(58)]
    lens[0] = min(lens[0], most)
    s = Setup(74, fmt, 1, 16, 8, d, 64, lens, cols=4096 // 64)
    q = s.rows(len(lens), 16)
    out, lse = attend(s, q, [1] * len(lens), 0.1, max_len=most)
    check_attention(s, q, [1] * len(lens), out, lse, 0.1, only=[0, 1, 2, 3, 30, 61], heads=[0, 7])


@by_fmt
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("case", ["few", "tiny", "mixed", "long", "drafts", "many", "more"])
def test_attention_in_shares(gpu_lib, case, d, fmt):
    """Decoding calls whose work is divided on the device: pairs that lie in one workgroup's share, begin or end in it, or span
    several, sequences without tokens, rows or a range that counts among them, batches of more than 64 sequences, and of
    more than the division takes."""
    rng = np.random.default_rng(91)
    Hq, Hkv, page, only, bound = 4, 2, 64, None, 1 << 19
    if case == "few":
        lens, new = [1, 33, 4000], [1, 1, 1]
    elif case == "tiny":
        lens, new = [int(n) for n in rng.integers(0, 40, 130)], [1] * 130
    elif case == "mixed":
        lens, new = [0, 1500, 17, 0, 0, 2900, 1, 31, 32, 33, 700, 0, 64], [1, 1, 0, 1, 0, 1, 1, 1, 1, 1, 1, 1, 0]
    elif case == "long":
        lens, new, Hkv, Hq = [30011, 5], [1, 1], 1, 2
    elif case == "drafts":
        lens, new, Hq = [5, 900, 0, 3100, 40, 2, 64], [8, 3, 2, 7, 0, 4, 1], 6  # three query heads a KV head: 24 rows
    elif case == "many":
        lens = [int(n) for n in rng.integers(0, 90, 300)]
        lens[77], lens[201], lens[299] = 2500, 1200, 800
        new, only = [1] * 300, [0, 1, 63, 64, 76, 77, 78, 128, 200, 201, 202, 298, 299]
    else:
        lens = [int(n) for n in rng.integers(0, 20, 1030)]
        lens[3], lens[1029] = 5000, 4100  # in chunks
        new, Hkv, Hq, only, bound = [1] * 1030, 1, 1, [0, 3, 4, 500, 1028, 1029], 1 << 16
    s = Setup(92, fmt, 1, Hq, Hkv, d, page, lens, cols=bound // page)
    q = s.rows(max(sum(new), 1), Hq)
    step = B.Step(q.shape[1], max(new), torch.from_numpy(offsets_of(new)).cuda())
    ws = torch.full((B.tp_cache8_workspace_size(s.dims, s.cache, step, bound),), 0xFF, dtype=torch.uint8, device="cuda")  # NaN
    assert ws.numel() > 0
    out, lse = attend(s, q, new, 0.1, max_len=bound, ws=ws)
    check_attention(s, q, new, out, lse, 0.1, only=only)
    again, l2 = attend(s, q, new, 0.1, max_len=bound, ws=ws)
    assert torch.equal(out, again) and torch.equal(lse, l2)
    # the bound that the sequences need: the same within the tolerance
    out, lse = attend(s, q, new, 0.1, max_len=max(max(lens), 1))
    check_attention(s, q, new, out, lse, 0.1, only=only)


@pytest.mark.parametrize("heads", [(2, 1), (8, 4)])
def test_attention_in_shares_of_many_sequences(gpu_lib, heads):
    """The most sequences that are divided on the device, most of them short, a long one first, last and beside others."""
    rng = np.random.default_rng(94)
    lens = [int(n) for n in rng.integers(0, 70, 1024)]
    lens[0], lens[511], lens[512], lens[1023] = 3000, 900, 4000, 2000
    s = Setup(95, c.FP8, 1, *heads, 64, 64, lens, cols=1 << 10)
    q = s.rows(1024, heads[0])
    out, lse = attend(s, q, [1] * 1024, 0.1, max_len=1 << 16)
    check_attention(s, q, [1] * 1024, out, lse, 0.1, only=[0, 1, 2, 510, 511, 512, 513, 700, 1022, 1023])
    again, l2 = attend(s, q, [1] * 1024, 0.1, max_len=1 << 16)
    assert torch.equal(out, again) and torch.equal(lse, l2)


@by_fmt
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("case", ["tokens", "drafts", "prompts"])
def test_attention_of_several_layers_split(gpu_lib, case, d, fmt):
    """Several layers in a call that is divided (one and two tiles of rows) or planned in chunks (four): a pair over many
    shares, several pairs in one, sequences without tokens; queries and outputs with the layers inside a token's rows."""
    L, Hkv, bound = 3, 2, 1 << 16
    lens = [30011, 0, 700] + [(7 * i) % 40 for i in range(40)] + [2100]
    only = [0, 1, 2, 3, 20, 42, 43]
    if case == "tokens":
        Hq, new = 4, [1] * 44
    elif case == "drafts":
        Hq, new = 6, [3, 1, 8] + [1 + i % 5 for i in range(40)] + [2]  # up to 24 rows
    else:
        L, lens, only, Hq, new, bound = 2, [9000, 40, 700], None, 16, [9, 1, 4], 1 << 14  # up to 72
    s = Setup(96, fmt, L, Hq, Hkv, d, 64, lens, cols=bound // 64)
    total = sum(new) + 1
    q = s.rows(total, Hq)
    out, lse = attend(s, q, new, 0.1, max_len=bound)
    check_attention(s, q, new, out, lse, 0.1, only=only)
    assert bool((out[:, -1] == -7).all()) and bool((lse[:, :, -1] == -7).all())
    step = B.Step(total, max(new), torch.from_numpy(offsets_of(new)).cuda())
    inside = bf16(q).cuda().transpose(0, 1).contiguous()  # [total][L][Hq][d]
    got, l2 = torch.full_like(inside, -7.0), torch.full_like(lse, -7.0)
    B.tp_cache8_attention(s.dims, s.cache, step, inside.transpose(0, 1), 0.1, bound, got.transpose(0, 1), l2)
    assert torch.equal(got.transpose(0, 1), out) and torch.equal(l2, lse)
    for l in range(L):  # a call for each layer alone, on its part of the pages
        dims = B.dims(1, Hq, Hkv, d)
        one = B.Cache8(dims, s.dev[l], s.dtable, s.lens, 64, fmt)
        alone, l1 = torch.full_like(out[l], -7.0), torch.full_like(lse[l], -7.0)
        B.tp_cache8_attention(dims, one, step, bf16(q[l]).cuda(), 0.1, bound, alone, l1)
        s1 = Setup.__new__(Setup)
        s1.__dict__.update(s.__dict__, L=1, pages=s.pages[l:l + 1])
        check_attention(s1, q[l:l + 1], new, alone[None], l1[None], 0.1, only=[0, 2])


def test_attention_in_shares_with_bad_ranges(gpu_lib):
    """Ranges and lengths that do not count have no blocks; the pairs behind them keep their places."""
    lens = [700, 900, 50, 600, 2000, 64]
    s = Setup(93, c.INT, 1, 4, 2, 64, 32, lens, cols=1 << 14)
    s.lens_ = [700, 900, 50, 600, 10 ** 9, 64]  # (10^9 counts as 0)
    s.upload()
    off = [0, 2, 99, 2, 4, 5, -1]  # 1: leaves the rows, 2 and 5: fall
    q = s.rows(6, 4)
    out = torch.full((6, 4, 64), -7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((4, 6), -7.0, device="cuda")
    B.tp_cache8_attention(s.dims, s.cache, B.Step(6, 2, torch.tensor(off, dtype=torch.int32, device="cuda")), bf16(q[0]).cuda(), 0.1,
                          1 << 19, out, lse)
    out, lse = f64(out), f64(lse)
    for b, rows in ((0, [0, 1]), (3, [2, 3])):
        for t, row in enumerate(rows):
            for hq in range(4):
                k, v, there = s.held(b, 0, hq // 2, lens[b])
                bound = cc.bounds(q[0, row, hq], k, v, there & (np.arange(lens[b]) <= lens[b] - 2 + t), 0.1)
                assert cc.accepts(out[row, hq], lse[hq, row], bound), (b, row, hq)
    assert not out[4].any() and np.all(lse[:, 4] == -math.inf)
    assert np.all(out[5] == -7) and np.all(lse[:, 5] == -7)


@by_fmt
def test_attention_strides(gpu_lib, fmt):
    """Queries inside a fused projection's rows, head-major queries and outputs, an output between guards, one query for all."""
    s = Setup(34, fmt, 1, 8, 2, 64, 32, [90, 41])
    new, scale = [3, 2], 0.125
    q = s.rows(5, 8)
    want, wl = attend(s, q, new, scale)
    fused = torch.randn((5, 14, 64), device="cuda").to(torch.bfloat16)
    fused[:, 2:10] = bf16(q[0]).cuda()
    guarded = torch.full((5, 11, 72), -7.0, dtype=torch.bfloat16, device="cuda")
    step = B.Step(5, 3, torch.tensor([0, 3, 5], dtype=torch.int32, device="cuda"))
    B.tp_cache8_attention(s.dims, s.cache, step, fused[:, 2:10], scale, 96, guarded[:, 1:9, :64])
    assert torch.equal(guarded[:, 1:9, :64], want[0])
    guarded[:, 1:9, :64] = -7.0
    assert bool((guarded == -7).all())
    heads = bf16(q[0]).cuda().transpose(0, 1).contiguous()  # [Hq][total][d]
    out = torch.empty_like(heads)
    B.tp_cache8_attention(s.dims, s.cache, step, heads.transpose(0, 1), scale, 96, out.transpose(0, 1), wl)
    assert torch.equal(out.transpose(0, 1), want[0])
    one = bf16(q[0, :1, :1]).cuda()
    out = torch.empty((5, 8, 64), dtype=torch.bfloat16, device="cuda")
    B.tp_cache8_attention(s.dims, s.cache, step, one.expand(5, 8, 64), scale, 96, out)
    alike, _ = attend(s, np.broadcast_to(q[:, :1, :1], q.shape).copy(), new, scale)
    assert torch.equal(out, alike[0])


@by_fmt
@pytest.mark.parametrize("lens,new", [([90, 41], [3, 2]), ([9000, 70], [17, 1]), ([300], [100]), ([2000, 0], [1, 1])])
def test_attention_in_place(gpu_lib, lens, new, fmt):
    """Outputs on the queries' memory, with one to four tiles of rows, whole and in chunks."""
    s = Setup(42, fmt, 1, 8, 2, 128, 64, lens)
    q = s.rows(sum(new), 8)
    rows, lse = bf16(q).cuda(), torch.full((1, 8, sum(new)), -7.0, device="cuda")
    step = B.Step(sum(new), max(new), torch.from_numpy(offsets_of(new)).cuda())
    B.tp_cache8_attention(s.dims, s.cache, step, rows, 0.1, max(lens), rows, lse)
    check_attention(s, q, new, rows, lse, 0.1)


@by_fmt
def test_one_token_without_offsets_and_padded_batch(gpu_lib, fmt):
    """offsets = NULL: row b is sequence b's token; padded sequences have length 0, rows behind the batch stay."""
    s = Setup(35, fmt, 1, 8, 2, 128, 64, [100, 0, 33, 0], cols=2)
    q = s.rows(6, 8)
    out = torch.full((6, 8, 128), -7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((8, 6), -7.0, device="cuda")
    B.tp_cache8_attention(s.dims, s.cache, B.Step(6), bf16(q[0]).cuda(), 0.1, 128, out, lse)
    check_attention(s, q, [1, 1, 1, 1], out[None], lse[None], 0.1)
    assert bool((out[4:] == -7).all()) and bool((lse[:, 4:] == -7).all())
    k, v = s.rows(6, 2), s.rows(6, 2)
    B.tp_cache8_append(s.dims, s.cache, B.Step(6), bf16(k[0]).cuda(), bf16(v[0]).cuda())
    append_expected(s, s.lens_, [1] * 4, [0, 1, 2, 3, 4], k, v, np.zeros((1, 6, 8, 128)), None, None, 0, 0)
    s.check_pages()


@by_fmt
def test_pool_beyond_4_gib(gpu_lib, fmt):
    """Pages whose offset passes 32 bits."""
    d, page, Hkv = 128, 256, 8
    dims = B.dims(1, 8, Hkv, d)
    each = B.tp_cache8_page_bytes(dims, page) * Hkv
    num = (1 << 32) // each + 40
    small = Setup(36, fmt, 1, 8, Hkv, d, page, [600, 20])
    pool = torch.zeros(num * each, dtype=torch.uint8, device="cuda").view(num, Hkv, page // 32, -1)
    at = torch.arange(num - small.num, num, device="cuda")
    pool[at] = small.dev[0]
    table = torch.where(small.dtable >= 0, small.dtable + (num - small.num), -1).to(torch.int32)
    big = B.Cache8(dims, pool, table, small.lens, page, fmt)
    q, k, v = (bf16(small.rows(2, 8)[0]).cuda() for _ in range(3))
    outs = []
    for cache in (small.cache, big):
        B.tp_cache8_append(dims, cache, B.Step(2), k, v)
        out = torch.empty((2, 8, d), dtype=torch.bfloat16, device="cuda")
        B.tp_cache8_attention(dims, cache, B.Step(2), q, 0.1, 768, out)
        kk = torch.empty((1, Hkv, 620, d), dtype=torch.bfloat16, device="cuda")
        vv = torch.empty_like(kk)
        B.tp_cache8_read(dims, cache, B.Batch([0, 600, 620]), kk, vv)
        outs.append((out, kk, vv))
    assert all(torch.equal(a, b) for a, b in zip(*outs))
    assert torch.equal(pool[at], small.dev[0]) and not bool(pool[:num - small.num].any())


@by_fmt
def test_largest_batch(gpu_lib, fmt):
    """65535 sequences of one token, every page its own: attention gives each its value back."""
    n = 65535
    dims = B.dims(1, 2, 1, 64)
    pages = torch.full((n * B.tp_cache8_page_bytes(dims, 32),), 0xFF, dtype=torch.uint8, device="cuda")
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    table = torch.randperm(n, device="cuda", generator=g).to(torch.int32).view(n, 1)
    cache = B.Cache8(dims, pages, table, torch.ones(n, dtype=torch.int32, device="cuda"), 32, fmt)
    k, v = (torch.randn((n, 1, 64), device="cuda", generator=g).to(torch.bfloat16) for _ in range(2))
    q = torch.randn((n, 2, 64), device="cuda", generator=g).to(torch.bfloat16)
    B.tp_cache8_append(dims, cache, B.Step(n), k, v)
    out, lse = torch.full_like(q, -7.0), torch.zeros((2, n), device="cuda")
    B.tp_cache8_attention(dims, cache, B.Step(n), q, 0.125, 32, out, lse)
    scale = v.double().abs().amax(-1, keepdim=True) / c.qmax(fmt)
    # half a step of the code, one weight rounded to fp16 and divided by in fp32 (2^-10.9), and bf16's 2^-8
    step = scale / 2 if fmt == c.INT else torch.maximum(v.double().abs() * 2.0 ** -4, scale * 2.0 ** -10)
    assert bool(((out.double() - v.double()).abs() <= step * 1.01 + v.double().abs() * 1.07 * (2.0 ** -8 + 2.0 ** -10.8)).all())


@by_fmt
def test_shared_pages(gpu_lib, fmt):
    """A prefix that sequences share is listed by all of them; a page may also come twice in one sequence."""
    s = Setup(77, fmt, 1, 8, 2, 128, 32, [200, 200, 96, 64])
    s.table[1, :5] = s.table[0, :5]
    s.table[2, 2] = s.table[2, 0]
    s.upload()
    q = s.rows(4, 8)
    q[0, 1] = q[0, 0]
    out, lse = attend(s, q, [1] * 4, 0.1)
    check_attention(s, q, [1] * 4, out, lse, 0.1)


# ------------------------------------------------------------------------------ together
@pytest.mark.parametrize("fmt,bits", [(B.TP_QFMT_INT, 8), (B.TP_QFMT_INT, 6), (B.TP_QFMT_FP8_E4M3, 8)])
def test_evict_load_decode_read_evict(gpu_lib, fmt, bits):
    """The way it is used: an eviction's compact cache into pages, decode steps, the answer read back and evicted again
    with the kept tokens."""
    L, Hq, Hkv, d, lens, budget, steps = 2, 8, 2, 64, [300, 150], 50, 20
    rng = np.random.default_rng(41)
    dims = B.dims(L, Hq, Hkv, d)
    n, scale = sum(lens), 0.125
    k, v = (bf16(rng.normal(size=(L, Hkv, n, d))).cuda() for _ in range(2))
    qg = bf16(rng.normal(size=(L, Hq, 16, d))).cuda()
    batch = B.Batch([0, 300, 450], [0, 8, 16])
    kw = dict(softmax_scale=scale, pool_k=5, qfmt=fmt, bits=bits, keep_budget=budget)
    bufs = B.evict_fused(dims, batch, qg, k, v, **kw)
    s = Setup(42, fmt, L, Hq, Hkv, d, 32, [budget + steps] * 2)
    kept = bufs.kept_offsets
    B.tp_cache8_load(dims, s.cache, kept, bufs.k_c, bufs.v_q_c, bufs.scales_c, bits)
    kc = f64(bufs.k_c).reshape(L, Hkv, kept[-1], d)
    codes = bufs.v_q_c.cpu().numpy().reshape(L, Hkv, kept[-1], d) ^ (0 if fmt == c.FP8 else 128)
    sc = bufs.scales_c.cpu().numpy().reshape(L, Hkv, kept[-1])
    for b in range(2):
        for l in range(L):
            for h in range(Hkv):
                s.write(b, 0, l, h, {t: kc[l, h, kept[b] + t] for t in range(budget)},
                        {t: (codes[l, h, kept[b] + t], sc[l, h, kept[b] + t]) for t in range(budget)})
    s.check_pages()
    cs = table_of(400, d)
    rope = B.Rope(torch.from_numpy(cs).cuda(), d)
    for i in range(steps):
        s.lens_ = [budget + i + 1] * 2
        s.lens.copy_(torch.tensor(s.lens_, dtype=torch.int32))
        pos = np.array([300 + i, 150 + i], dtype=np.int32)
        qn, kn, vn = s.rows(2, Hq), s.rows(2, Hkv), s.rows(2, Hkv)
        qr = bf16(qn).cuda()
        B.tp_cache8_append(dims, s.cache, B.Step(2), bf16(kn).cuda(), bf16(vn).cuda(), torch.from_numpy(pos).cuda(), rope, qr, qr)
        out = torch.empty((L, 2, Hq, d), dtype=torch.bfloat16, device="cuda")
        lse = torch.empty((L, Hq, 2), device="cuda")
        B.tp_cache8_attention(dims, s.cache, B.Step(2), qr, scale, budget + steps, out, lse)
        want = append_expected(s, s.lens_, [1, 1], [0, 1, 2], kn, vn, qn, cs, pos, d, 0)
        s.check_pages()
        same(f64(qr), want)
        check_attention(s, want, [1, 1], out, lse, scale)
    m = budget + steps
    k2 = torch.empty((L, Hkv, 2 * m, d), dtype=torch.bfloat16, device="cuda")
    v2 = torch.empty_like(k2)
    back = B.Batch([0, m, 2 * m], [0, 8, 16])
    B.tp_cache8_read(dims, s.cache, back, k2, v2)
    for b in range(2):
        kk, vv, _ = s.held(b, 1, 0, m)
        same(f64(k2[1, 0, b * m:(b + 1) * m]), c4.by_fp32(kk))
        same(f64(v2[1, 0, b * m:(b + 1) * m]), c4.by_fp32(vv))
    kw["keep_budget"] = 20
    again = B.evict_fused(dims, back, qg, k2, v2, **kw)
    idx = again.kept_idx.view(L, Hkv, 40).cpu().numpy()
    assert np.all(np.diff(idx[..., :20]) > 0) and idx.min() >= 0 and idx.max() < m
    B.tp_cache8_load(dims, s.cache, again.kept_offsets, again.k_c, again.v_q_c, again.scales_c, bits)
    s.lens.fill_(20)
    k3 = torch.empty((L, Hkv, 40, d), dtype=torch.bfloat16, device="cuda")
    v3 = torch.empty_like(k3)
    B.tp_cache8_read(dims, s.cache, B.Batch([0, 20, 40]), k3, v3)
    was = again.k_c.view_as(k3).double()
    # half a step of a scale of at most the largest / Q, or 2^-4 of the number; then bf16's 2^-8
    most = was.abs().max() / c.qmax(fmt) / 2 if fmt == c.INT else torch.maximum(was.abs() * 2.0 ** -4, was.abs().max() / 448 * 2.0 ** -10)
    assert bool(((k3.double() - was).abs() <= most * 1.01 + k3.double().abs() * 2.0 ** -8).all())


@by_fmt
def test_captured_steps_with_shared_workspace(gpu_lib, fmt):
    """Two captured decode steps of different sequences on one workspace, replayed with lengths, positions and tokens
    changed in place, against eager calls; the program's own work between the replays."""
    setups = [Setup(51 + i, fmt, 1, 8, 2, 128, 64, [900, 1, 300], cols=16, spare=40) for i in range(2)]
    for s in setups:  # pages for growth
        free = [p for p in range(s.num) if p not in s.table]
        for b in range(3):
            for i in range(s.table.shape[1]):
                if s.table[b, i] < 0 and free:
                    s.table[b, i] = free.pop()
        s.upload()
    dims, step = setups[0].dims, B.Step(3)
    rope = B.Rope(torch.from_numpy(table_of(3000, 128)).cuda(), 128)
    ws = torch.empty(B.tp_cache8_workspace_size(dims, setups[0].cache, step, 1024), dtype=torch.uint8, device="cuda")
    io = []
    for s in setups:
        t = {n: torch.zeros((3, h, 128), dtype=torch.bfloat16, device="cuda") for n, h in (("q", 8), ("k", 2), ("v", 2), ("qr", 8), ("o", 8))}
        t["pos"], t["lse"] = torch.zeros(3, dtype=torch.int32, device="cuda"), torch.zeros((8, 3), device="cuda")
        io.append(t)

    def call(t, cache):
        B.tp_cache8_append(dims, cache, step, t["k"], t["v"], t["pos"], rope, t["q"], t["qr"])
        B.tp_cache8_attention(dims, cache, step, t["qr"], 0.1, 1024, t["o"], t["lse"], ws)

    side = torch.cuda.Stream()
    graphs = []
    for s, t in zip(setups, io):
        with torch.cuda.stream(side):
            call(t, s.cache)
        side.synchronize()
        s.dev.copy_(torch.from_numpy(s.pages))
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            call(t, s.cache)
        graphs.append(g)
    rng = np.random.default_rng(53)
    for i in range(4):
        for s, t, g in zip(setups, io, graphs):
            s.lens.add_(1)
            for n in ("q", "k", "v"):
                t[n].copy_(bf16(rng.normal(size=t[n].shape) * 1.5 ** i))
            t["pos"].copy_(torch.from_numpy(rng.integers(0, 3000, 3).astype(np.int32)))
            copy = s.dev.clone()
            g.replay()
            torch.cuda.synchronize()
            got = [t[n].clone() for n in ("qr", "o", "lse")] + [s.dev.clone()]
            for n in ("qr", "o", "lse"):
                t[n].zero_()
            call(t, B.Cache8(dims, copy, s.dtable, s.lens, 64, fmt))
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, [t["qr"], t["o"], t["lse"], copy])), i
            s.pages = copy.cpu().numpy()
            s.lens_ = s.lens.tolist()
            check_attention(s, f64(t["qr"])[None], [1, 1, 1], t["o"][None], t["lse"][None], 0.1)


def test_two_streams(gpu_lib):
    """Two calls at once on streams of their own read one cache, each with its workspace."""
    s = Setup(61, c.INT, 1, 8, 2, 64, 32, [3000, 500])
    q = [s.rows(2, 8) for _ in range(2)]
    want = [attend(s, x, [1, 1], 0.125) for x in q]
    step, streams = B.Step(2), [torch.cuda.Stream() for _ in range(2)]
    dev = [bf16(x[0]).cuda() for x in q]
    outs = [torch.zeros((2, 8, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(10):
        for st, x, out in zip(streams, dev, outs):
            B.tp_cache8_attention(s.dims, s.cache, step, x, 0.125, 3008, out, stream=st)
    torch.cuda.synchronize()
    for out, (w, _) in zip(outs, want):
        assert torch.equal(out, w[0])


@pytest.mark.parametrize("how", ["stream", "handle", "default"])
def test_scratch_of_the_calls_stream(gpu_lib, monkeypatch, how):
    """Without a workspace, on a stream that is not the current one: the scratch is that stream's, and the current
    stream's pending work keeps the memory that it uses."""
    s = Setup(71, c.FP8, 1, 8, 2, 64, 32, [3000, 500])
    q = s.rows(2, 8)
    want, lse = attend(s, q, [1, 1], 0.125)
    mine, other = torch.cuda.Stream(), torch.cuda.Stream()
    on = {"stream": other, "handle": other, "default": torch.cuda.default_stream()}[how]
    given = {"stream": other, "handle": other.cuda_stream, "default": 0}[how]
    rows, out, l = bf16(q[0]).cuda(), torch.zeros_like(want[0]), torch.zeros_like(lse[0])
    need = B.tp_cache8_workspace_size(s.dims, s.cache, B.Step(2), 3008)
    assert need > 0
    torch.cuda.synchronize()
    empty, made = torch.empty, []

    def spy(*size, **kw):
        made.append(torch.cuda.current_stream().cuda_stream)
        return empty(*size, **kw)

    with torch.cuda.stream(mine):
        big = torch.ones(64 << 20, device="cuda")
        held = torch.full((need,), 3, dtype=torch.uint8, device="cuda")
        kept = held
        for _ in range(20):
            big.mul_(1.0)
        kept = held.clone()  # queued behind the products; the block is free for this stream's next allocation
        del held
        monkeypatch.setattr(torch, "empty", spy)
        B.tp_cache8_attention(s.dims, s.cache, B.Step(2), rows, 0.125, 3008, out, l, stream=given)
        monkeypatch.undo()
        assert torch.cuda.current_stream() == mine
    torch.cuda.synchronize()
    assert made == [on.cuda_stream]
    assert torch.equal(out, want[0]) and torch.equal(l, lse[0])
    assert bool((kept == 3).all())


@pytest.mark.parametrize("given", ["current", "stream", "handle"])
def test_captured_without_a_workspace(gpu_lib, given):
    """A captured call that makes its own scratch, on the capturing stream: replays against eager calls."""
    s = Setup(79, c.INT, 1, 8, 2, 64, 32, [3000, 500])
    side, step = torch.cuda.Stream(), B.Step(2)
    rows, out = torch.zeros((2, 8, 64), dtype=torch.bfloat16, device="cuda"), torch.zeros((2, 8, 64), dtype=torch.bfloat16, device="cuda")
    stream = {"current": None, "stream": side, "handle": side.cuda_stream}[given]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        B.tp_cache8_attention(s.dims, s.cache, step, rows, 0.125, 3008, out, stream=stream)
    for i in range(4):
        q = s.rows(2, 8)
        rows.copy_(bf16(q[0]))
        want, _ = attend(s, q, [1, 1], 0.125)
        other = [torch.full((1 << 20,), i, device="cuda") for _ in range(3)]  # the program's own memory
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[0])
        assert all(bool((x == i).all()) for x in other)


def test_captured_step_follows_its_lengths(gpu_lib):
    """One captured call for lengths from 0 to its bound: every replay is that of the lengths that the tensor holds, also
    where the division into shares changes."""
    bound = 1 << 15
    s = Setup(80, c.FP8, 1, 4, 1, 128, 64, [9000, 700, 3, 5000], cols=bound // 64)
    q = s.rows(4, 4)
    rows = bf16(q[0]).cuda()
    out, lse = torch.zeros((4, 4, 128), dtype=torch.bfloat16, device="cuda"), torch.zeros((4, 4), device="cuda")
    ws = torch.empty(B.tp_cache8_workspace_size(s.dims, s.cache, B.Step(4), bound), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        B.tp_cache8_attention(s.dims, s.cache, B.Step(4), rows, 0.1, bound, out, lse, ws)
    for lens in ([9000, 700, 3, 5000], [1, 0, 0, 2], [0, 0, 0, 0], [33, 700, 1, 4999], [9000, 0, 3, 1]):
        s.lens_ = lens
        s.lens.copy_(torch.tensor(lens, dtype=torch.int32))
        ws.fill_(0xFF)
        out.fill_(-7.0)
        graph.replay()
        torch.cuda.synchronize()
        check_attention(s, q, [1] * 4, out[None], lse[None], 0.1)


def test_formats_do_not_mix(gpu_lib):
    """A handle of one width is refused by the other's calls."""
    s4 = T.Setup(62, 1, 2, 2, 64, 32, [5])
    s8 = Setup(62, c.INT, 1, 2, 2, 64, 32, [5])
    q = bf16(s8.rows(1, 2)[0]).cuda()
    for d, cache, attention, append in ((s4.dims, s4.cache, B.tp_cache8_attention, B.tp_cache8_append),
                                        (s8.dims, s8.cache, B.tp_cache_attention, B.tp_cache_append)):
        with pytest.raises(ValueError):
            attention(d, cache, B.Step(1), q, 0.1, 32, torch.empty_like(q))
        with pytest.raises(ValueError):
            append(d, cache, B.Step(1), q, q)
    with pytest.raises(ValueError):
        B.Cache8(s8.dims, s8.dev, s8.dtable, s8.lens, 32, 2)
