"""What tp_cache8_attention allocates, it allocates on the stream that the call runs on (no GPU: the stand-ins of
test_binding_streams.py)."""
import types

import pytest

from paper_2608_03276_amd import binding as B
from test_binding_streams import DIMS, Tensor, made  # noqa: F401 (the fixture)


@pytest.mark.parametrize("stream,handle", [(None, None), (types.SimpleNamespace(cuda_stream=0x1230), 0x1230), (0x1230, 0x1230),
                                           (0, 0)], ids=["current", "stream", "handle", "default"])
def test_scratch_is_made_on_the_calls_stream(made, monkeypatch, stream, handle):  # noqa: F811
    monkeypatch.setattr(B, "_cache8_call", lambda d, cache, tensors, s: B._stream(s))
    monkeypatch.setattr(B, "_rows", lambda *args: B.TpRows())
    monkeypatch.setattr(B, "_on_device", lambda *args: None)
    c = B.TpCache8(B.TpCache(0x10000, 0x10000, 0x10000, 400, 64, 200, 2), 0)
    cache = types.SimpleNamespace(c=c, ref=B.ctypes.byref(c), device="cpu", index=0, batch=2)
    B.tp_cache8_attention(DIMS, cache, B.Step(2), Tensor(), 0.1, 10000, Tensor(), None, None, stream)
    assert made and all(h == handle for h in made)
