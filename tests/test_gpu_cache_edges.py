"""The paged 4-bit cache on the GPU: streams, ranges and shapes at the edges of the contracts, against the float64
oracle.  Tolerances are those of test_gpu_cache.py where nothing else is said."""
import math

import numpy as np
import pytest
import torch

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
