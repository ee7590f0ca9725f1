"""Buffers that the harness allocates for a call on another stream are not handed to the current one while the call runs."""
import numpy as np
import pytest
import torch

from paper_2605_17170_amd import harness
from paper_2605_17170_amd import workloads as wl
from test_gpu_shared import build

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("handle", [False, True])
@pytest.mark.parametrize("shared", [False, True])
def test_buffers_of_a_call_on_a_busy_stream(shared, handle):
    from oracle import tkv_oracle
    tkv_oracle.build()
    cache, _, _ = build(101, [900], [30, 130], 2)
    try:
        n = 1 if shared else 0
        q = harness.bf16_tensor(wl.make_q(np.random.SeedSequence([101, 5]), 3 - n, 8), DEV)
        if shared:
            cache.plan_shared([[0, 1]], 8, 8, 8)
        else:
            cache.plan_decode(8)
        call = cache.decode_shared if shared else cache.decode
        want = call(q).clone()
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            torch.cuda._sleep(50_000_000)          # some 20 ms: what follows is queued behind it
        out = call(q, stream=side.cuda_stream if handle else side)
        held = [torch.full((size,), 0x5A, dtype=torch.uint8, device=DEV) for size in (1 << 10, 1 << 13, 1 << 15, 1 << 17, 1 << 19, 1 << 21) for _ in range(4)]
        torch.cuda.synchronize()
        assert torch.equal(out, want) and all(bool((t == 0x5A).all()) for t in held)
    finally:
        cache.close()
