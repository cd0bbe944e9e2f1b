"""The paged cache's entry points on the CPU: sizes, and every refusal that the header names (no call here
reaches a launch; the tests skip where a GPU is visible)."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2608_03276_amd import binding as B

lib = B.load()
no_gpu = pytest.mark.skipif(torch.cuda.device_count() > 0, reason="validation cases use fake device pointers")
FAKE = 0x10000
D = B.dims(2, 8, 2, 128)


def cache(pages=FAKE, table=FAKE, lens=FAKE, num=10, tokens=64, cols=5, batch=3):
    return B.TpCache(pages, table, lens, num, tokens, cols, batch)


def step(offsets=FAKE, total=7, most=4):
    return B.TpStep(offsets, total, most)


def rows(data=FAKE, layer=0, token=1024, head=128):
    return B.TpRows(data, layer, token, head)


def ref(x):
    return None if x is None else ctypes.byref(x)


def out_rows(**kw):
    return rows(**{"layer": 7 * 1024, **kw})


def test_page_bytes():
    for d, each in ((64, 72), (128, 140)):
        for t in (32, 64, 128, 256):
            assert B.tp_cache_page_bytes(B.dims(1, 8, 2, d), t) == t * each
    for d, t in ((B.dims(1, 8, 2, 96), 64), (B.dims(1, 8, 3, 64), 64), (B.dims(1, 8, 2, 64), 48), (B.dims(1, 8, 2, 64), 512)):
        assert lib.tp_cache_page_bytes(ctypes.byref(d), t) == 0
        assert lib.tp_last_error().decode() != ""
    assert lib.tp_cache_page_bytes(None, 64) == 0


CACHES = [(None, B.TP_ERR_NULL), (cache(pages=None), B.TP_ERR_NULL), (cache(table=None), B.TP_ERR_NULL),
          (cache(pages=FAKE + 8), B.TP_ERR_PARAM), (cache(table=FAKE + 2), B.TP_ERR_PARAM),
          (cache(lens=FAKE + 1), B.TP_ERR_PARAM), (cache(tokens=16), B.TP_ERR_UNSUPPORTED),
          (cache(tokens=96), B.TP_ERR_UNSUPPORTED), (cache(tokens=0), B.TP_ERR_UNSUPPORTED),
          (cache(num=0), B.TP_ERR_SHAPE), (cache(cols=0), B.TP_ERR_SHAPE), (cache(batch=0), B.TP_ERR_SHAPE),
          (cache(batch=65536), B.TP_ERR_UNSUPPORTED), (cache(num=2 ** 31), B.TP_ERR_UNSUPPORTED),
          (cache(tokens=256, cols=2 ** 22 + 1), B.TP_ERR_UNSUPPORTED)]


def _load(c=cache(), ko=(0, 5, 5, 300), k=FAKE, vq=FAKE, sc=FAKE, bits=4, d=D):
    return lib.tp_cache_load(ref(d), ref(c), None if ko is None else B._i64_array(ko), k, vq, sc, bits, None)


def _append(c=cache(), s=step(), k=rows(), v=rows(), pos=FAKE, rope=B.TpRope(FAKE, 100, 128, 0), q=None, qo=None, d=D):
    return lib.tp_cache_append(ref(d), ref(c), ref(s), ref(k), ref(v), pos, ref(rope), ref(q), ref(qo), None)


def _attend(c=cache(), s=step(), q=rows(), scale=0.1, most=320, o=out_rows(), lse=FAKE, ws=FAKE, wsb=1 << 40, d=D):
    return lib.tp_cache_attention(ref(d), ref(c), ref(s), ref(q), scale, most, ref(o), lse, ws, wsb, None)


def _read(c=cache(), off=(0, 5, 5, 300), first=None, k=FAKE, v=FAKE, d=D, batch=True):
    bt = B.Batch(off) if batch else None
    return lib.tp_cache_read(ref(d), ref(c), ref(bt.c) if bt else None, None if first is None else B._i64_array(first),
                             k, v, None)


@no_gpu
@pytest.mark.parametrize("call", [_load, _append, _attend, _read])
def test_cache_and_dims_refusals(call):
    for c, want in CACHES:
        assert call(c=c) == want, (want, c and [getattr(c, f[0]) for f in c._fields_])
        assert lib.tp_last_error().decode() != ""
    assert call(d=None) == B.TP_ERR_NULL
    assert call(d=B.dims(1, 8, 2, 96)) == B.TP_ERR_UNSUPPORTED
    assert call(d=B.dims(1, 8, 3, 64)) == B.TP_ERR_SHAPE
    if call is not _load:  # the lengths are needed
        assert call(c=cache(lens=None)) == B.TP_ERR_NULL


@no_gpu
def test_load_refusals():
    assert _load(ko=None) == B.TP_ERR_NULL
    assert _load(ko=(1, 5, 5, 300)) == B.TP_ERR_SHAPE
    assert _load(ko=(0, 5, 4, 300)) == B.TP_ERR_SHAPE
    assert _load(ko=(0, 5, 5, 326)) == B.TP_ERR_SHAPE  # 321 tokens, 320 in the pages
    assert _load(k=None) == _load(vq=None) == _load(sc=None) == B.TP_ERR_NULL
    assert _load(k=FAKE + 8) == _load(vq=FAKE + 4) == _load(sc=FAKE + 4) == B.TP_ERR_PARAM
    assert _load(bits=1) == _load(bits=9) == B.TP_ERR_PARAM
    assert _load(bits=5) == _load(bits=8) == B.TP_ERR_UNSUPPORTED
    assert _load(c=cache(batch=65), ko=[0] * 66) == B.TP_ERR_UNSUPPORTED
    assert _load(c=cache(tokens=256, cols=2 ** 22), ko=(0, 0, 0, 2 ** 30), d=B.dims(1, 8, 2, 64)) == B.TP_ERR_UNSUPPORTED
    assert _load(c=cache(lens=None), ko=(0, 0, 0, 0)) == B.TP_OK  # nothing to do, and no lengths needed


STEPS = [(None, B.TP_ERR_NULL), (step(total=0), B.TP_ERR_SHAPE), (step(most=0), B.TP_ERR_SHAPE),
         (step(offsets=None, total=3, most=2), B.TP_ERR_SHAPE), (step(offsets=None, total=2, most=1), B.TP_ERR_SHAPE),
         (step(offsets=FAKE + 2), B.TP_ERR_PARAM)]
ROWS = [(None, B.TP_ERR_NULL), (rows(data=None), B.TP_ERR_NULL), (rows(data=FAKE + 8), B.TP_ERR_PARAM),
        (rows(token=1028), B.TP_ERR_PARAM), (rows(head=-128), B.TP_ERR_PARAM), (rows(layer=4), B.TP_ERR_PARAM),
        (rows(token=2 ** 59), B.TP_ERR_UNSUPPORTED)]
OVERLAPS = [out_rows(head=64), out_rows(token=1016), out_rows(layer=1024), out_rows(layer=0), out_rows(token=0),
            rows(layer=1024, token=2048, head=64)]


@no_gpu
def test_append_refusals():
    for s, want in STEPS:
        assert _append(s=s) == want
    for r, want in ROWS:
        assert _append(k=r) == _append(v=r) == want
        if r is not None:  # NULL with q_out is a NULL of the pair
            assert _append(q=r, qo=out_rows()) == _append(q=rows(), qo=r) == want
    for r in OVERLAPS:
        assert _append(q=rows(), qo=r) == B.TP_ERR_SHAPE
    assert _append(q=rows()) == _append(qo=out_rows()) == B.TP_ERR_NULL
    assert _append(rope=None, q=rows(), qo=out_rows()) == B.TP_ERR_NULL
    assert _append(q=out_rows(), qo=out_rows(layer=8 * 1024)) == B.TP_ERR_SHAPE  # q's memory at other strides
    assert _append(pos=None) == B.TP_ERR_NULL
    assert _append(pos=FAKE + 2) == B.TP_ERR_PARAM
    for rope, want in [((None, 100, 128, 0), B.TP_ERR_NULL), ((FAKE + 4, 100, 128, 0), B.TP_ERR_PARAM),
                       ((FAKE, 0, 128, 0), B.TP_ERR_SHAPE), ((FAKE, 100, 128, 2), B.TP_ERR_PARAM),
                       ((FAKE, 100, 0, 0), B.TP_ERR_PARAM), ((FAKE, 100, 24, 1), B.TP_ERR_PARAM),
                       ((FAKE, 100, 144, 0), B.TP_ERR_PARAM)]:
        assert _append(rope=B.TpRope(*rope)) == want, rope
    assert _append(s=step(total=2 ** 31 - 1, most=2 ** 31 - 1)) == B.TP_ERR_UNSUPPORTED


@no_gpu
def test_attention_refusals():
    for s, want in STEPS:
        assert _attend(s=s) == want
    for r, want in ROWS:
        assert _attend(q=r) == want
        assert _attend(o=r) == want
    for r in OVERLAPS:
        assert _attend(o=r) == B.TP_ERR_SHAPE
    assert _attend(q=out_rows(), o=out_rows(layer=8 * 1024)) == B.TP_ERR_SHAPE  # q's memory at other strides
    for scale in (0.0, -1.0, float("inf"), float("nan"), 3e38):
        assert _attend(scale=scale) == B.TP_ERR_PARAM
    assert _attend(most=0) == _attend(most=321) == B.TP_ERR_SHAPE
    assert _attend(lse=FAKE + 2) == B.TP_ERR_PARAM
    wide = cache(cols=64)  # 4096 tokens: partial results of several chunks
    n = ctypes.c_size_t(0)
    assert lib.tp_cache_workspace_size(ref(D), ref(wide), ref(step()), 4096, ctypes.byref(n)) == B.TP_OK and n.value > 0
    for kw in (dict(ws=None), dict(wsb=0), dict(ws=FAKE + 16), dict(wsb=n.value - 1)):
        assert _attend(c=wide, most=4096, **kw) == B.TP_ERR_WORKSPACE, kw
    assert lib.tp_cache_workspace_size(ref(D), ref(cache()), ref(step()), 320, None) == B.TP_ERR_NULL
    assert lib.tp_cache_workspace_size(ref(D), ref(cache()), ref(step()), 321, ctypes.byref(n)) == B.TP_ERR_SHAPE
    big = step(total=2 ** 31 - 1, most=2 ** 31 - 1)
    assert _attend(s=big) == B.TP_ERR_UNSUPPORTED


@no_gpu
def test_read_refusals():
    assert _read(batch=False) == B.TP_ERR_NULL
    assert _read(off=(0, 5, 5)) == B.TP_ERR_SHAPE  # two sequences for a cache of three
    assert _read(off=(0, 5, 4, 300)) == B.TP_ERR_SHAPE
    assert _read(k=None) == _read(v=None) == B.TP_ERR_NULL
    assert _read(k=FAKE + 8) == _read(v=FAKE + 2) == B.TP_ERR_PARAM
    assert _read(first=(0, -1, 0)) == B.TP_ERR_SHAPE
    assert _read(first=(0, 0, 2 ** 30 - 294)) == B.TP_ERR_SHAPE
    assert _read(off=(0, 0, 0, 2 ** 62)) == B.TP_ERR_SHAPE
    assert _read(c=cache(batch=65), off=[0] * 66) == B.TP_ERR_UNSUPPORTED
    assert _read(off=(0, 0, 0, 0)) == B.TP_OK


def test_workspace_size_never_falls():
    """A buffer sized for the longest call serves the others of the same dims."""
    def size(d, batch, total, most, length):
        n = ctypes.c_size_t(0)
        c = B.TpCache(FAKE, FAKE, FAKE, 10, 256, 2 ** 20, batch)
        assert lib.tp_cache_workspace_size(ref(d), ref(c), ref(B.TpStep(FAKE, total, most)), length, ctypes.byref(n)) == B.TP_OK
        return n.value

    rng = np.random.default_rng(3)
    for _ in range(3000):
        hkv = int(rng.choice([1, 2, 8]))
        d = B.dims(int(rng.choice([1, 1, 4, 32])), hkv * int(rng.choice([1, 4, 8])), hkv, int(rng.choice([64, 128])))
        batch, most, length = (int(np.exp(rng.uniform(0, np.log(x)))) for x in (300, 3000, 300000))
        total = int(rng.integers(most, batch * most + 1))
        grown = [batch, total, most, length]
        i = int(rng.integers(0, 4))
        grown[i] = int(grown[i] * np.exp(rng.uniform(0, 1.5))) + 1
        if grown[2] > grown[1]:
            grown[1] = grown[2]
        assert size(d, batch, total, most, length) <= size(d, *grown), (batch, total, most, length, grown)
    assert size(B.dims(1, 8, 2, 64), 64, 64, 1, 128) == 0  # one chunk: no partial results


def test_binding_checks():
    """What the binding refuses by itself, on tensors of the wrong kind (CPU tensors here)."""
    with pytest.raises(ValueError):
        B.Cache(D, torch.zeros(64 * 140 * 4, dtype=torch.uint8), torch.zeros((1, 1), dtype=torch.int32), None, 64)
    with pytest.raises(ValueError):
        B.Step(3, 1, torch.zeros(4, dtype=torch.int32))
    with pytest.raises(ValueError):
        B.Rope(torch.zeros((4, 64)), 64)
    with pytest.raises(B.TaskPressError):
        B.tp_cache_page_bytes(D, 100)
