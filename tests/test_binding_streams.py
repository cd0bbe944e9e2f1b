"""The binding allocates what a call writes on the stream that the call runs on: a block of another stream's pool may
still be in use by what is queued there.  No GPU: the entry points, torch's streams and its allocation are stand-ins
that record where an allocation was made."""
import contextlib
import types

import pytest
import torch

from paper_2608_03276_amd import binding as B

DIMS = B.dims(1, 8, 2, 64)
BATCH = B.Batch([0, 40, 100], [0, 4, 8])


class Tensor:
    """A device tensor of any size."""

    is_cuda, device, dtype = True, "cpu", torch.bfloat16

    def is_contiguous(self):
        return True

    def numel(self):
        return 1 << 40

    def element_size(self):
        return 1

    def data_ptr(self):
        return 0x10000


class Library:
    """The host-only entry points as they are, the others without effect."""

    def __init__(self, lib):
        self.lib = lib

    def __getattr__(self, name):
        if name in ("tp_workspace_size", "tp_cache_workspace_size", "tp_keep_count", "tp_last_error"):
            return getattr(self.lib, name)
        return lambda *args: 0


@pytest.fixture
def made(monkeypatch):
    """The handles of the streams that were current at each allocation (None: the caller's)."""
    library, empty, current, out = Library(B.load()), torch.empty, [None], []

    @contextlib.contextmanager
    def stream(s):
        current.append(s.cuda_stream)
        yield
        current.pop()

    def spy(*size, **kw):
        out.append(current[-1])
        return empty(1, dtype=kw.get("dtype"))

    monkeypatch.setattr(B, "load", lambda: library)
    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle, device=None: types.SimpleNamespace(cuda_stream=handle))
    monkeypatch.setattr(torch.cuda, "default_stream", lambda device=None: types.SimpleNamespace(cuda_stream=0))
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: types.SimpleNamespace(cuda_stream=77))
    monkeypatch.setattr(torch, "empty", spy)
    monkeypatch.setattr(B, "_need", lambda *args, **kw: None)
    return out


def cache_attention(monkeypatch, stream):
    monkeypatch.setattr(B, "_cache_call", lambda d, cache, tensors, s: B._stream(s))
    monkeypatch.setattr(B, "_rows", lambda *args: B.TpRows())
    monkeypatch.setattr(B, "_on_device", lambda *args: None)
    c = B.TpCache(0x10000, 0x10000, 0x10000, 400, 64, 200, 2)
    cache = types.SimpleNamespace(c=c, ref=B.ctypes.byref(c), device="cpu", index=0, batch=2)
    B.tp_cache_attention(DIMS, cache, B.Step(2), Tensor(), 0.1, 10000, Tensor(), None, None, stream)


t = Tensor()
CALLS = {
    "tp_cache_attention": cache_attention,
    "tp_guide_attention": lambda m, s: B.tp_guide_attention(DIMS, BATCH, t, t, t, 0.1, t, t, None, s),
    "tp_guide_attention_quantize": lambda m, s: B.tp_guide_attention_quantize(DIMS, BATCH, t, t, t, 0.1, B.TP_QFMT_INT, 4, t, t,
                                                                             t, t, None, s),
    "tp_combine_select_topk": lambda m, s: B.tp_combine_select_topk(DIMS, BATCH, t, t, 0, 0.0, 8, [0, 8, 16], t, None, None, s),
    "evict": lambda m, s: B.evict(DIMS, BATCH, t, t, t, softmax_scale=0.1, pool_k=5, qfmt=B.TP_QFMT_INT, bits=4, keep_budget=8,
                                  stream=s),
    "evict_fused": lambda m, s: B.evict_fused(DIMS, BATCH, t, t, t, softmax_scale=0.1, pool_k=5, qfmt=B.TP_QFMT_INT, bits=4,
                                              keep_budget=8, stream=s),
}


@pytest.mark.parametrize("call", CALLS.values(), ids=CALLS)
@pytest.mark.parametrize("stream,handle", [(None, None), (types.SimpleNamespace(cuda_stream=0x1230), 0x1230), (0x1230, 0x1230),
                                           (0, 0)], ids=["current", "stream", "handle", "default"])
def test_buffers_are_made_on_the_calls_stream(made, monkeypatch, call, stream, handle):
    call(monkeypatch, stream)
    assert made and all(h == handle for h in made)
