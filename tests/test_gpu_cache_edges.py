"""The paged 4-bit cache on the GPU: streams, ranges and shapes at the edges of the contracts, against the float64
oracle.  Tolerances are those of test_gpu_cache.py where nothing else is said."""
import math

import numpy as np
import pytest
import torch

import cache_cases as cc
import test_gpu_cache as T
from oracle import cache_oracle as c
from paper_2608_03276_amd import binding as B

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------ streams
@pytest.mark.parametrize("how", ["stream", "handle", "default"])
def test_scratch_of_the_calls_stream(gpu_lib, monkeypatch, how):
    """Without a workspace, on a stream that is not the current one: the scratch is that stream's, and the current
    stream's pending work keeps the memory that it uses."""
    s = T.Setup(71, 1, 8, 2, 64, 32, [3000, 500])
    q = s.rows(2, 8)
    want, lse = T.attend(s, q, [1, 1], 0.125)
    mine, other = torch.cuda.Stream(), torch.cuda.Stream()
    on = {"stream": other, "handle": other, "default": torch.cuda.default_stream()}[how]
    given = {"stream": other, "handle": other.cuda_stream, "default": 0}[how]
    rows, out, l = T.bf16(q[0]).cuda(), torch.zeros_like(want[0]), torch.zeros_like(lse[0])
    need = B.tp_cache_workspace_size(s.dims, s.cache, B.Step(2), 3008)
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
        B.tp_cache_attention(s.dims, s.cache, B.Step(2), rows, 0.125, 3008, out, l, stream=given)
        monkeypatch.undo()
        assert torch.cuda.current_stream() == mine
    torch.cuda.synchronize()
    assert made == [on.cuda_stream]
    assert torch.equal(out, want[0]) and torch.equal(l, lse[0])
    assert bool((kept == 3).all())


# ------------------------------------------------------------------------------ scores that fp32 does not hold
@pytest.mark.parametrize("n", [90, 700, 9000])
@pytest.mark.parametrize("T_", [1, 6, 12, 20])
@pytest.mark.parametrize("d", [64, 128])
def test_attention_scores_beyond_fp32(gpu_lib, d, T_, n):
    """A row with a score of +infinity or NaN has no softmax: o and lse are NaN, not those of a row that sees nothing.
    A score of -infinity is a key that is not seen.  The rows beside it keep their results.

    Ordinary rows: a group's |q| sums to 26 * 2^-62 (at most 40 here) under scales of 2^60, so delta of test_gpu_cache.py is
    4 * 40/4 * 72 * 7 * 2^-24 = 2^-9.7 for these; 2^-10 of the log-sum-exp holds with 26, 2^-10.9 + 2 delta + 2^-14 is 2^-8.5."""
    s = T.Setup(72, 1, 4, 2, d, 64, [n])
    blocks = s.pages.reshape(-1, 2, s.page // 32, c.block_bytes(d))  # [page][head][block]
    blocks[..., :16 * d].reshape(*blocks.shape[:3], 32, 4, d // 32, 4)[..., 0, :] = 0xFF  # channels 0..31: codes 7
    ks = c.bf16_bits(np.full((*blocks.shape[:3], 32, d // 32), 2.0 ** 60))
    ks[:, 1, :, ::3] = 0  # head 1: every third key is zero
    blocks[..., 32 * d:34 * d] = ks.reshape(*blocks.shape[:3], -1).view(np.uint8)
    s.upload()
    kinds = ["ordinary", "up", "down", "nan", "inf", "both"]
    q = s.rows(T_, 4) * 2.0 ** -62
    for t in range(T_):
        kind = kinds[(t + 1) % 6] if T_ > 1 else "up"
        if kind in ("up", "down", "both"):
            q[0, t] = 0.0
            q[0, t, :, :32] = {"up": 1, "down": -1, "both": 1}[kind] * 2.0 ** 70
            if kind == "both":  # the two heads of a KV head: one row up, one ordinary
                q[0, t, ::2] = s.rows(1, 4)[0, 0, ::2] * 2.0 ** -62
    q = c.to_bf16(q)
    finite = q.copy()
    for t in range(T_):
        kind = kinds[(t + 1) % 6] if T_ > 1 else "up"
        if kind in ("nan", "inf"):
            q[0, t, :, 5] = np.nan if kind == "nan" else np.inf
    out, lse = T.attend(s, q, [T_], 1.0)
    out, lse = T.f64(out)[0], T.f64(lse)[0]
    held = [c.held(s.pages, d, s.table[0], s.page, 0, h, n) for h in range(2)]
    for t in range(T_):
        kind = kinds[(t + 1) % 6] if T_ > 1 else "up"
        for h in range(4):
            tag, got, l = (kind, t, h), out[t, h], lse[h, t]
            if kind in ("up", "nan", "inf") or (kind == "both" and h % 2 == 1):
                assert np.isnan(l) and np.isnan(got).all(), (tag, l, got[:4])
            elif kind == "down" and h < 2:  # every score is -infinity
                assert l == -math.inf and not got.any(), (tag, l)
            elif kind == "down":            # the zero keys' mean
                v = held[1][1][:n - T_ + t + 1:1]
                v = v[np.abs(held[1][0][:len(v)]).max(1) == 0]
                assert abs(l - math.log(len(v))) <= 2.0 ** -13, (tag, l)
                tol = np.abs(v).mean(0) * (2.0 ** -10.9 + 2.0 ** -14) + 2.0 ** -8 * np.abs(v.mean(0)) + n * 2.0 ** -30 * np.abs(v).max()
                assert np.all(np.abs(got - v.mean(0)) <= tol), tag
            else:
                k, v, _ = held[h // 2]
                ref, want, mag = c.attend(finite[0, t, h], k, v, np.arange(n) <= n - T_ + t, 1.0)
                assert abs(l - want) <= 2.0 ** -10, (tag, l, want)
                assert np.all(np.abs(got - ref) <= mag * 2.0 ** -8.5 + 2.0 ** -8 * np.abs(ref) + n * 2.0 ** -30 * np.abs(v).max()), tag


@pytest.mark.parametrize("lens,new", [([1, 70], [1, 1]), ([1, 700], [1, 20]), ([33, 9000], [5, 6])])
@pytest.mark.parametrize("d", [64, 128])
def test_attention_scores_of_any_size(gpu_lib, d, lens, new):
    """Rows whose keys all have one score, of magnitudes from 1 to 2^40: their mean up to 2^26 / log2(e), beyond that as for
    infinities.  The scores are exact; the log-sum-exp's error is 2^-22 of it and of the score, and 2^-14."""
    s = T.Setup(70, 1, 4, 2, d, 64, lens)
    blocks = s.pages.reshape(-1, c.block_bytes(d))
    words = blocks[:, :16 * d].reshape(len(blocks), 32, 4, d // 32, 4)
    words[:] = 0x88
    words[:, :, 0, 0, 0] = 0x8C  # channel 0: 4
    blocks[:, 32 * d:34 * d] = c.bf16_bits(np.full((len(blocks), d), 0.25)).view(np.uint8).reshape(len(blocks), -1)
    s.upload()
    held = [[c.held(s.pages, d, s.table[b], 64, 0, h, lens[b])[1] for h in range(2)] for b in range(2)]
    for x in (1.0, 2.0 ** 20, 1.375 * 2.0 ** 25, 1.40625 * 2.0 ** 25, 1.5 * 2.0 ** 25, 2.0 ** 31, 1.125 * 2.0 ** 37, 2.0 ** 40):
        for sign in (1, -1):
            q = np.zeros((1, sum(new), 4, d))
            q[..., 0] = sign * x
            out, lse = T.attend(s, q, new, 1.0)
            out, lse = T.f64(out)[0], T.f64(lse)[0]
            far = x * 1.4426950408889634 > 2.0 ** 26
            for row in range(sum(new)):
                b, t = (0, row) if row < new[0] else (1, row - new[0])
                n = lens[b] - new[b] + t + 1
                for h in range(4):
                    tag, got, l = (sign * x, b, t, h), out[row, h], lse[h, row]
                    if far and sign > 0:
                        assert np.isnan(l) and np.isnan(got).all(), (tag, l)
                    elif far:
                        assert l == -math.inf and not got.any(), (tag, l)
                    else:
                        v = held[b][h // 2][:n]
                        mean, mag = v.mean(0), np.abs(v).mean(0)
                        want = sign * x + math.log(n)
                        assert abs(l - want) <= 2.0 ** -21 * x + 2.0 ** -14 + 2.0 ** -22 * abs(want), (tag, l, want)
                        tol = mag * (2.0 ** -10.9 + 2.0 ** -14) + 2.0 ** -8 * np.abs(mean) + n * 2.0 ** -30 * np.abs(v).max()
                        assert np.all(np.abs(got - mean) <= tol), tag


def test_attention_of_a_far_first_block(gpu_lib):
    """A block all of whose keys score far below 0, before ordinary ones, leaves nothing behind."""
    s = T.Setup(69, 1, 4, 2, 128, 64, [40, 700])
    q, scale = cc.fill(s, "massive", 2)
    blocks = s.pages.reshape(-1, 2, s.page // 32, c.block_bytes(128))
    for page, j in ((s.table[0, 0], 0), (s.table[1, 0], 0), (s.table[1, 3], 1)):
        for h in range(2):
            blk = blocks[page, h, j]
            blk[:16 * 128].reshape(32, 4, 4, 4)[:] = 0x88
            blk[:16 * 128].reshape(32, 4, 4, 4)[:, 0, 0, 0] = 0x81
            blk[32 * 128:34 * 128] = c.bf16_bits(np.full(128, 2.0 ** 45)).view(np.uint8)
    s.upload()
    out, lse = T.attend(s, q, [1, 1], scale, max_len=700)
    out, lse = T.f64(out)[0], T.f64(lse)[0]
    for row, hq, bound in cc.rows(s, [1, 1], q, scale):
        assert cc.accepts(out[row, hq], lse[hq, row], bound), (row, hq, lse[hq, row], bound[1])


# ------------------------------------------------------------------------------ key scales
@pytest.mark.parametrize("shape", range(len(cc.SHAPES)))
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kind", cc.KINDS)
def test_attention_contents(gpu_lib, kind, d, shape):
    """Strong and weak groups of channels, blocks of different power, tokens of very large keys, scores far from 0: within
    what the arithmetic allows (cache_cases.py), for each form of the kernel."""
    Hq, Hkv, lens, new, most = cc.SHAPES[shape]
    s = T.Setup(80 + shape, 1, Hq, Hkv, d, 64, lens)
    q, scale = cc.fill(s, kind, sum(new))
    s.upload()
    out, lse = T.attend(s, q, new, scale, max_len=most)
    out, lse = T.f64(out)[0], T.f64(lse)[0]
    for row, hq, bound in cc.rows(s, new, q, scale):
        ref, want, tol, tol_lse = bound
        assert cc.accepts(out[row, hq], lse[hq, row], bound), (
            row, hq, float(np.max(np.abs(out[row, hq] - ref) / np.maximum(tol, 1e-300))), lse[hq, row], want, tol_lse)


# ------------------------------------------------------------------------------ streamed caches
@pytest.mark.parametrize("R,T_", [(1, 1), (8, 4), (8, 5)])
def test_attention_of_a_large_cache_of_small_heads(gpu_lib, R, T_):
    """d = 64 and a length bound by which the cache is streamed, with one to four tiles."""
    lens, new = [9000, 700, 17, 5000], [T_, min(T_, 2), T_, 1]
    s = T.Setup(73, 1, 2 * R, 2, 64, 64, lens, cols=1 << 14)
    q = s.rows(sum(new), 2 * R)
    out, lse = T.attend(s, q, new, 0.1, max_len=1 << 20, max_new=T_)
    T.check_attention(s, q, new, T.f64(out), T.f64(lse), 0.1, heads=[1])
    few, lse_few = T.attend(s, q, new, 0.1, max_len=9000, max_new=T_)
    T.check_attention(s, q, new, T.f64(few), T.f64(lse_few), 0.1, heads=[1])


@pytest.mark.parametrize("most", [4096, 2048])
def test_attention_of_many_whole_sequences(gpu_lib, most):
    """Eight waves a sequence, streamed (496 pairs of up to 4096 tokens are 284 MB) and not."""
    lens = [2500, 4, 0, 700] + [1 + i % 40 for i in range(58)]
    lens[0] = min(lens[0], most)
    s = T.Setup(74, 1, 16, 8, 128, 64, lens, cols=4096 // 64)
    q = s.rows(len(lens), 16)
    out, lse = T.attend(s, q, [1] * len(lens), 0.1, max_len=most)
    T.check_attention(s, q, [1] * len(lens), T.f64(out), T.f64(lse), 0.1, only=[0, 1, 2, 3, 30, 61], heads=[0, 7])


# ------------------------------------------------------------------------------ outputs on the queries, a second eviction
@pytest.mark.parametrize("lens,new", [([90, 41], [3, 2]), ([9000, 70], [17, 1]), ([300], [100]), ([2000, 1], [1, 1])])
@pytest.mark.parametrize("d", [64, 128])
def test_attention_in_place_is_right(gpu_lib, d, lens, new):
    """Outputs written over the queries, whole and in chunks, against the oracle."""
    s = T.Setup(75, 1, 8, 2, d, 64, lens)
    q = s.rows(sum(new), 8)
    rows, lse = T.bf16(q[0]).cuda(), torch.full((8, sum(new)), -7.0, device="cuda")
    step = B.Step(sum(new), max(new), torch.from_numpy(T.offsets_of(new)).cuda())
    B.tp_cache_attention(s.dims, s.cache, step, rows, 0.1, max(lens), rows, lse)
    got, gl = T.f64(rows), T.f64(lse)
    for row, hq, bound in cc.rows(s, new, q, 0.1):
        assert cc.accepts(got[row, hq], gl[hq, row], bound), (row, hq)


def codes_and_scales(s, b, layer, head, n):
    """Codes and scales of a sequence's first n tokens: keys int [n][d], float [n][d / 32], values int [n][d], float [n]."""
    d, out = s.d, [[], [], [], []]
    pages = s.dev.cpu().numpy()
    kb, ks, vb, vs = c.places(d)
    for t in range(0, n, 32):
        page, j, _ = c.place_of(s.table[b], s.num, s.page, t)
        block = pages[layer, page, head, j]
        bits = block[32 * d:34 * d].copy().view(np.uint16).astype(np.uint32) << 16
        for part, x in zip(out, ((block[kb] >> ks & 15).astype(int) - 8, bits.view(np.float32).reshape(32, -1),
                                 (block[vb] >> vs & 15).astype(int) - 8, block[34 * d:].copy().view(np.float32))):
            part.append(x)
    return [np.concatenate(x)[:n].astype(np.float64) for x in out]


@pytest.mark.parametrize("d,page", [(64, 32), (128, 64)])
def test_second_eviction_keeps_the_codes(gpu_lib, d, page):
    """Rows read back, evicted again and loaded: the kept tokens' codes are those that were held.  A scale is 1/7 of the
    rounded 7 scale: off by at most 2^-8 of itself for values, by that and its own rounding, 2^-8 more, for keys (the
    largest code of a group or row is 7)."""
    L, Hq, Hkv, lens, budget = 2, 4, 2, [300, 77], [45, 45]
    s = T.Setup(76, L, Hq, Hkv, d, page, lens)
    n = sum(lens)
    step = B.Step(n, max(lens), torch.from_numpy(T.offsets_of(lens)).cuda())
    B.tp_cache_append(s.dims, s.cache, step, T.bf16(s.rows(n, Hkv, 3.0)).cuda(), T.bf16(s.rows(n, Hkv, 0.2)).cuda())
    before = {(b, l, h): codes_and_scales(s, b, l, h, lens[b]) for b in range(2) for l in range(L) for h in range(Hkv)}
    k = torch.empty((L, Hkv, n, d), dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    back = B.Batch([0, 300, 377], [0, 8, 16])
    B.tp_cache_read(s.dims, s.cache, back, k, v)
    qg = T.bf16(s.rng.normal(size=(L, Hq, 16, d))).cuda()
    bufs = B.evict_fused(s.dims, back, qg, k, v, softmax_scale=0.125, pool_k=5, qfmt=B.TP_QFMT_INT, bits=4, keep_budget=45)
    B.tp_cache_load(s.dims, s.cache, bufs.kept_offsets, bufs.k_c, bufs.v_q_c, bufs.scales_c, 4)
    idx = bufs.kept_idx.view(L, Hkv, 90).cpu().numpy()
    for (b, l, h), was in before.items():
        kept = idx[l, h, 45 * b:45 * (b + 1)]
        now = codes_and_scales(s, b, l, h, 45)
        assert np.array_equal(now[0], was[0][kept]) and np.array_equal(now[2], was[2][kept]), (b, l, h)
        assert np.all(np.abs(now[1] / was[1][kept] - 1) <= 2.0 ** -7 * (1 + 2.0 ** -8)), (b, l, h)
        assert np.all(np.abs(now[3] / was[3][kept] - 1) <= 2.0 ** -8 * (1 + 2.0 ** -8)), (b, l, h)


# ------------------------------------------------------------------------------ batches, pages, captured calls
def test_largest_batch(gpu_lib):
    """65535 sequences of one token, every page its own: attention gives each its value back, bit for bit as read."""
    n = 65535
    dims = B.dims(1, 2, 1, 64)
    pages = torch.zeros(n * B.tp_cache_page_bytes(dims, 32), dtype=torch.uint8, device="cuda")
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    table = torch.randperm(n, device="cuda", generator=g).to(torch.int32).view(n, 1)
    cache = B.Cache(dims, pages, table, torch.ones(n, dtype=torch.int32, device="cuda"), 32)
    k, v = (torch.randn((n, 1, 64), device="cuda", generator=g).to(torch.bfloat16) for _ in range(2))
    q = torch.randn((n, 2, 64), device="cuda", generator=g).to(torch.bfloat16)
    B.tp_cache_append(dims, cache, B.Step(n), k, v)
    out, lse = torch.full_like(q, -7.0), torch.zeros((2, n), device="cuda")
    B.tp_cache_attention(dims, cache, B.Step(n), q, 0.125, 32, out, lse)
    few = [0, 1, 31, 4095, 40000, 65471, 65534]
    back = B.Cache(dims, pages, table[few].contiguous(), torch.ones(len(few), dtype=torch.int32, device="cuda"), 32)
    kk, vv = (torch.empty((1, 1, len(few), 64), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    B.tp_cache_read(dims, back, B.Batch(list(range(len(few) + 1))), kk, vv)
    held = vv[0, 0].float()
    for h in range(2):  # one weight, rounded to fp16 once and divided by in fp32: 2^-11, and bf16's 2^-8
        assert bool(((out[few, h].float() - held).abs() <= held.abs() * (2.0 ** -8 + 2.0 ** -10.9)).all())
        want = 0.125 * (q[few, h].float() * kk[0, 0].float()).sum(1)
        # keys read back are rounded to bf16: 2^-8 of each of 64 terms, of at most 3 * 4 * 0.125 each
        assert bool(((lse[h, few] - want).abs() <= 64 * 1.5 * 2.0 ** -8).all())
    scale = (v.float().abs().amax(-1, keepdim=True) / 7)
    assert bool(((out.float() - v.float()).abs() <= scale * (0.5 + 7 * 2.0 ** -7)).all())  # every row: half a step


def test_shared_pages(gpu_lib):
    """A prefix that sequences share is listed by all of them; a page may also come twice in one sequence."""
    s = T.Setup(77, 1, 8, 2, 128, 32, [200, 200, 96, 64])
    s.table[1, :5] = s.table[0, :5]
    s.table[2, 2] = s.table[2, 0]
    s.upload()
    q = s.rows(4, 8)
    q[0, 1] = q[0, 0]
    out, lse = T.attend(s, q, [1] * 4, 0.1)
    got, gl = T.f64(out)[0], T.f64(lse)[0]
    for row, hq, bound in cc.rows(s, [1] * 4, q, 0.1):
        assert cc.accepts(got[row, hq], gl[hq, row], bound), (row, hq)


@pytest.mark.parametrize("d", [64, 128])
def test_load_leaves_out_missing_pages(gpu_lib, d):
    s = T.Setup(78, 2, 2, 2, d, 32, [100, 64, 33])
    s.table[0, 1], s.table[1, 0], s.table[2, 1] = -1, s.num, 2 ** 31 - 1
    s.upload()
    off = [0, 100, 164, 197]
    k = c.to_bf16(s.rng.normal(size=(2, 2, 197, d)))
    v = T.bf16(s.rng.normal(size=(2, 2, 197, d))).cuda()
    scales = torch.empty((2, 2, 197), device="cuda")
    v_q = torch.empty((2, 2, 197, d // 2), dtype=torch.uint8, device="cuda")
    B.tp_quantize_v_scales(s.dims, B.Batch([0, 197]), v, B.TP_QFMT_INT, 4, scales, v_q)
    B.tp_cache_load(s.dims, s.cache, off, T.bf16(k).cuda(), v_q, scales, 4)
    vv = T.f64(v)
    for b in range(3):
        for t in range(off[b + 1] - off[b]):
            for l in range(2):
                for h in range(2):
                    s.write(b, t, l, h, c.quantise_key(k[l, h, off[b] + t]), c.quantise_value(vv[l, h, off[b] + t]))
    s.check_pages()


@pytest.mark.parametrize("given", ["current", "stream", "handle"])
def test_captured_without_a_workspace(gpu_lib, given):
    """A captured call that makes its own scratch, on the capturing stream: replays against eager calls."""
    s = T.Setup(79, 1, 8, 2, 64, 32, [3000, 500])
    side, step = torch.cuda.Stream(), B.Step(2)
    rows, out = torch.zeros((2, 8, 64), dtype=torch.bfloat16, device="cuda"), torch.zeros((2, 8, 64), dtype=torch.bfloat16, device="cuda")
    stream = {"current": None, "stream": side, "handle": side.cuda_stream}[given]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        B.tp_cache_attention(s.dims, s.cache, step, rows, 0.125, 3008, out, stream=stream)
    for i in range(4):
        q = s.rows(2, 8)
        rows.copy_(T.bf16(q[0]))
        want, _ = T.attend(s, q, [1, 1], 0.125)
        other = [torch.full((1 << 20,), i, device="cuda") for _ in range(3)]  # the program's own memory
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[0])
        assert all(bool((x == i).all()) for x in other)
