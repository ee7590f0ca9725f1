"""tkv_prefill_attention: a prefix that ends inside a tile of keys, with rows of another sequence, or of none, behind it."""
import math

import pytest
import torch

from tests.test_gpu_prefill import BF, DEV, FP, Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,most", [(32, 1 << 20), (32, 1), (128, 1 << 20), (128, 1), (256, 1 << 20), (256, 1)])
@pytest.mark.parametrize("heads", [1, 3])
@pytest.mark.parametrize("bad", [math.inf, math.nan])
@pytest.mark.parametrize("kv", [BF, FP])
def test_rows_behind_a_prefix_do_not_reach_it(rows, most, heads, bad, kv):
    for cached in (1, 2, 5, 15, 16, 17, 29, 31, 33, 47, 49, 63, 65, 70, 97, 113, 127, 129):
        c, clean = (Case([20, 30], [cached, 200], 2 * heads, heads, BF, kv, BF, seed=cached, kind=rows, most=most) for _ in range(2))
        clean.call()
        for x in c.before:
            x[cached:] = bad      # the second sequence's first rows stand behind the first one's last
        c.call()
        torch.cuda.synchronize()
        assert int(c.status.item()) == 0
        assert torch.equal(c.out[:20], clean.out[:20]), "%d rows of a prefix" % cached
        assert torch.isnan(c.out[20:]).all()


@pytest.mark.parametrize("rows", [32, 128, 256])
@pytest.mark.parametrize("bad", [math.inf, math.nan])
def test_rows_of_no_sequence_behind_the_last_prefix(rows, bad):
    for cached in (3, 30, 60, 100):
        c = Case([20], [cached], 4, 2, seed=cached, kind=rows)
        clean = c.out.clone()
        c.call()
        clean.copy_(c.out)
        c.before = [torch.cat([x, torch.full((100, 2, 128), bad, dtype=FP, device=DEV)]) for x in c.before]
        c.out.fill_(7.0)
        c.call()
        torch.cuda.synchronize()
        assert int(c.status.item()) == 0 and torch.equal(c.out, clean)
