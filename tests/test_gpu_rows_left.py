"""tkv_quantize_rows: rows of width 0 are their fp16 rounding, whatever they hold, in every place and beside rows of every width."""
import pytest
import torch

from paper_2605_17170_amd import tkv

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
SPECIAL = [float("inf"), float("-inf"), float("nan"), 1e30, -1e30, 65504.0, 65520.0, 1e-30, -0.0, 2.0 ** -24, 3e-8]


@pytest.mark.parametrize("heads", [1, 2, 5])
@pytest.mark.parametrize("bits", [2, 4])
@pytest.mark.parametrize("channel_keys", [False, True])
def test_rows_of_width_zero_are_rounded_and_nothing_else(heads, bits, channel_keys):
    n = 96
    g = torch.Generator(device=DEV)
    g.manual_seed(heads)
    x = [torch.randn((n, heads, 128), device=DEV, generator=g) for _ in range(2)]
    left = torch.arange(n, device=DEV) % 3 == 1                 # 32 rows, and 64 between them at `bits`
    for k, value in enumerate(SPECIAL):
        for part in range(2):
            rows = left.nonzero()[:, 0][k::len(SPECIAL)]
            x[part][rows, k % heads, (11 * k + part) % 128] = value
    x = [t.to(torch.bfloat16) for t in x]
    widths = torch.where(left, 0, bits).to(torch.uint8)
    blocks = None
    if channel_keys:
        blocks = (~left).nonzero()[:, 0].to(torch.int32).view(2, 32) if bits == 2 else torch.zeros((0, 32), dtype=torch.int32, device=DEV)
    out = [torch.full((n, heads, 128), 7.0, dtype=torch.float16, device=DEV) for _ in range(2)]
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    tkv.tkv_quantize_rows(tkv.tkv_desc.make(heads, 0, 0, int2_key_axis=1 if channel_keys else 0), *x, widths, blocks, *out, status)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    for o, t in zip(out, x):
        want = t[left].to(torch.float16)
        assert torch.equal(torch.isnan(o[left]), torch.isnan(want)) and torch.isnan(want).any()
        finite = ~torch.isnan(want)
        assert torch.equal(o[left].view(torch.int16)[finite], want.view(torch.int16)[finite])
        assert torch.isfinite(o[~left]).all()
