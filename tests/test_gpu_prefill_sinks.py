"""tkv_prefill_attention where one key has nearly all the weight and its value is small, so that the many others make the output.

Tolerance: in units of the row's largest weight, fp16 weights r are off by half a step, e = 2^-11 r, and by at most 2^-34 below 2^-23 (include/tkv.h); bf16
ones by 2^-8 r.  The output is off by at most sum e (|v| + |o|) / sum r.  Beside it, as in tests/prefill_model.py: the logits, summed in 32 bits, the
exponential, the sums over the keys, and the output's own half step."""
import math

import numpy as np
import pytest
import torch

from paper_2605_17170_amd import tkv
from tests.prefill_model import HALF, plan_of

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
SM = 1.0 / math.sqrt(128.0)
BF, FP = torch.bfloat16, torch.float16
GRID = 2.0 ** -34     # half of it, in units of the row's largest weight


def rows_of(n, sink, gap, spread, kind, seed):
    """Keys whose logits with a query of 16 in channel 0 lie `gap` below that of key `sink`, and values about 1, 0.02 at the sink."""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    k = torch.randn((n, 1, 128), device=DEV, generator=g)
    k[:, 0, 0] = torch.randn((n,), device=DEV, generator=g) * (spread / (16.0 * SM))
    k[sink, 0, 0] = gap / (16.0 * SM)
    v = 1.0 + 0.1 * torch.randn((n, 1, 128), device=DEV, generator=g)
    v[sink] = 0.02
    return k.to(kind), v.to(kind)


def exact(q, K, V, limits, half, out_type):
    """(value, tolerance) of query rows q [m, 128] that see the first `limits` keys each, in 64 bits.  half [n]: half a step of the keys' weights."""
    q, K, V = q.double(), K.double(), V.double()
    hidden = torch.arange(K.shape[0], device=DEV)[None] >= limits[:, None]
    logits = ((q @ K.t().contiguous()) * SM).masked_fill_(hidden, -math.inf)
    r = torch.exp(logits - logits.amax(-1, keepdim=True))
    total = r.sum(-1, keepdim=True)
    o, size = (r @ V) / total, (r @ V.abs()) / total
    e = torch.where(hidden, 0.0, torch.clamp(r * half, min=GRID))
    lost = (e @ V.abs() + e.sum(-1, keepdim=True) * o.abs()) / total
    off = (132 * 2.0 ** -24 * SM * (q.abs() @ K.abs().t().contiguous())).masked_fill_(hidden, 0.0).amax(-1, keepdim=True)
    rest = off + 2.0 ** -22 + K.shape[0] / 8 * 2.0 ** -23 + 16 * 2.0 ** -24
    return o, HALF[out_type] * o.abs() + 2.0 ** -25 + lost + rest * (size + o.abs())


def check(got, ref, tol, what):
    off = float(((got.double() - ref).abs() / tol).max())
    apart = float(((got.double() - ref).norm() / ref.norm()))
    print("  %s: %.3f of the tolerance, %.5f apart" % (what, off, apart), flush=True)
    assert off <= 1.0, "%s: %.3f of the tolerance" % (what, off)


@pytest.mark.parametrize("gap,spread", [(12.0, 0.5), (16.0, 0.0), (17.0, 0.0), (17.0, 0.5), (18.0, 0.0), (18.0, 0.5), (20.0, 0.5)])
@pytest.mark.parametrize("rows,most", [(32, 1 << 20), (32, 100), (128, 1 << 20), (128, 300), (256, 1 << 20)])
@pytest.mark.parametrize("q_type,kv_type", [(BF, BF), (BF, FP), (FP, FP)])
def test_a_sink_in_a_long_prefix(gap, spread, rows, most, q_type, kv_type):
    n, new, group = 60000, 3, 2
    for sink in (0, 41234):
        pk, pv = rows_of(n, sink, gap, spread, FP, int(gap))
        q = torch.zeros((new, group, 128), device=DEV).to(q_type)
        q[:, 0, 0], q[:, 1, 0] = 16.0, 15.5
        k = torch.zeros((new, 1, 128), device=DEV).to(kv_type)
        v = torch.ones((new, 1, 128), device=DEV).to(kv_type)
        desc = tkv.tkv_desc.make(1, 0, 0)
        plan = plan_of(rows, most, [new], [n], group)
        out = torch.zeros((new, group, 128), dtype=FP, device=DEV)
        ws = torch.zeros(max(16, tkv.tkv_prefill_workspace_bytes(desc, plan.n_slots, plan.tile_rows)), dtype=torch.uint8, device=DEV)
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        tkv.tkv_prefill_attention(desc, q, k, v, pk, pv, tkv.tkv_prefill.make(plan, DEV), SM, out, ws, status)
        torch.cuda.synchronize()
        assert int(status.item()) == 0
        K, V = torch.cat([pk[:, 0].double(), k[:, 0].double()]), torch.cat([pv[:, 0].double(), v[:, 0].double()])
        limits = torch.arange(n + 1, n + new + 1, device=DEV).repeat_interleave(group)
        half = torch.full((n + new,), HALF[FP], dtype=torch.float64, device=DEV)
        half[n:] = HALF[kv_type]
        ref, tol = exact(q.reshape(-1, 128), K, V, limits, half, FP)
        check(out.reshape(-1, 128), ref, tol, "gap %g, spread %g, sink %d, %d rows, ranges of %d" % (gap, spread, sink, rows, most))


@pytest.mark.parametrize("gap,spread", [(16.0, 0.0), (17.0, 0.5), (18.0, 0.5)])
@pytest.mark.parametrize("rows", [32, 128, 256])
def test_a_sink_among_the_new_tokens(gap, spread, rows):
    n, sink = 20000, 5
    k, v = rows_of(n, sink, gap, spread, FP, 3)
    q = torch.zeros((n, 1, 128), device=DEV).to(FP)
    q[:, 0, 0] = 16.0
    desc = tkv.tkv_desc.make(1, 0, 0)
    plan = plan_of(rows, 1 << 20, [n], [0], 1)
    out = torch.zeros((n, 1, 128), dtype=FP, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    tkv.tkv_prefill_attention(desc, q, k, v, None, None, tkv.tkv_prefill.make(plan, DEV), SM, out, None, status)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    at = torch.from_numpy(np.unique(np.round(np.geomspace(1, n, 200)).astype(np.int64)) - 1).to(DEV)
    ref, tol = exact(q[at, 0], k[:, 0], v[:, 0], at + 1, torch.full((n,), HALF[FP], dtype=torch.float64, device=DEV), FP)
    check(out[at, 0], ref, tol, "gap %g, spread %g, %d rows" % (gap, spread, rows))


@pytest.mark.parametrize("size", [2.0 ** 20, 2.0 ** 23, 2.0 ** 24, 2.0 ** 25])
@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("growth", [4, 8, 12, 16])
@pytest.mark.parametrize("rows,most", [(32, 1 << 20), (32, 3), (128, 1 << 20), (256, 1 << 20)])
def test_large_logits_that_grow_from_tile_to_tile(size, sign, growth, rows, most):
    """Logits (as powers of two) of about `size`, which 32-bit numbers hold in steps of up to 4; the largest of each 32 keys is `growth` above that
    of the 32 before, so that the reference lags behind as far as it may.  Weights stay finite and keep their ratios."""
    n = 640
    j = torch.arange(n, device=DEV)
    above = (j // 32 * growth + 1024 - torch.where(j % 32 == 7, 0, 512)).double()
    # a query of 2^14 in channel 0 and of 1 in channel 1: whole numbers, whose sum is exact in 32 bits
    k = torch.zeros((n, 1, 128), dtype=torch.float64, device=DEV)
    k[:, 0, 0], k[:, 0, 1] = sign * size / 2.0 ** 14, above
    q = torch.zeros((1, 1, 128), device=DEV).to(FP)
    q[0, 0, 0], q[0, 0, 1] = 2.0 ** 14, 1.0
    v = (j % 100).double()[:, None, None].expand(n, 1, 128).to(FP).contiguous()
    k = k.to(FP)
    sm = math.log(2.0)
    desc = tkv.tkv_desc.make(1, 0, 0)
    plan = plan_of(rows, most, [1], [n], 1)
    out = torch.zeros((1, 1, 128), dtype=FP, device=DEV)
    ws = torch.zeros(max(16, tkv.tkv_prefill_workspace_bytes(desc, plan.n_slots, plan.tile_rows)), dtype=torch.uint8, device=DEV)
    tkv.tkv_prefill_attention(desc, q, k[:1], v[:1], k, v, tkv.tkv_prefill.make(plan, DEV), sm, out, ws)
    torch.cuda.synchronize()
    K, V = torch.cat([k, k[:1]])[:, 0].double(), torch.cat([v, v[:1]])[:, 0].double()
    c = float(np.float32(sm) * np.float32(1.44269504088896340736))     # the call's factor, in 32 bits
    x = (K @ q[0, 0].double()) * c
    r = torch.exp2(x - x.max())
    o, size_of = (r @ V) / r.sum(), (r @ V.abs()) / r.sum()
    got = out[0, 0].double()
    assert torch.isfinite(got).all()
    # half a step of the weights and of the output; exponents of a few hundred at most, rounded to 32 bits: 2^-16 of a weight
    assert bool(((got - o).abs() <= 2.0 ** -11 * o.abs() + (2.0 ** -11 + 2.0 ** -16) * (size_of + o.abs())).all()), (got[0], o[0])
