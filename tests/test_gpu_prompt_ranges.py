"""Prompt attention, rows and distortion where offsets pass 32 bits: compared bit for bit with the same call on tensors of their own."""
import math

import numpy as np
import pytest
import torch

from paper_2605_17170_amd import tkv
from tests.prefill_model import plan_of

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
SM = 1.0 / math.sqrt(128.0)


def prefill(desc, q, k, v, before, plan, out):
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    ws = torch.empty(max(16, tkv.tkv_prefill_workspace_bytes(desc, plan.n_slots, plan.tile_rows)), dtype=torch.uint8, device=DEV)
    tkv.tkv_prefill_attention(desc, q, k, v, *before, tkv.tkv_prefill.make(plan, DEV), SM, out, ws, status)
    torch.cuda.synchronize()
    assert int(status.item()) == 0


@pytest.mark.parametrize("rows,most", [(32, 2), (128, 1 << 20), (256, 3)])
def test_prefixes_beyond_four_gigabytes(rows, most):
    hk, hq, old, new = 8, 16, [2200000, 301], [0, 9]
    desc = tkv.tkv_desc.make(hk, 0, 0)
    before = [torch.empty((sum(old), hk, 128), dtype=torch.float16, device=DEV) for _ in range(2)]
    for x in before:
        x[:1000] = math.nan
        x[-301:] = torch.randn((301, hk, 128), device=DEV).to(torch.float16)
    q, k, v = (torch.randn((9, h, 128), device=DEV).to(torch.bfloat16) for h in (hq, hk, hk))
    outs = [torch.zeros((9, hq, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    prefill(desc, q, k, v, before, plan_of(rows, most, new, old, hq // hk), outs[0])
    prefill(desc, q, k, v, [x[-301:].contiguous() for x in before], plan_of(rows, most, [9], [301], hq // hk), outs[1])
    assert torch.equal(*outs) and torch.isfinite(outs[0].float()).all()


def test_token_strides_beyond_two_gigabytes():
    n, stride = 600, 1 << 22
    desc = tkv.tkv_desc.make(1, 0, 0)
    wide = [torch.empty(n * stride, dtype=torch.bfloat16, device=DEV).as_strided((n, 1, 128), (stride, 128, 1)) for _ in range(3)]
    for x in wide:
        x.copy_(torch.randn((n, 1, 128), device=DEV))
    dense = [x.contiguous() for x in wide]
    for rows in (32, 128, 256):
        plan = plan_of(rows, 1 << 20, [n], [0], 1)
        outs = [torch.zeros((n, 1, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
        prefill(desc, *wide, [None, None], plan, outs[0])
        prefill(desc, *dense, [None, None], plan, outs[1])
        assert torch.equal(*outs)
    bits = torch.from_numpy(np.tile(np.array([0, 2, 4], np.uint8), n // 3)).to(DEV)
    got = []
    for K, V in ((wide[0], wide[1]), (dense[0], dense[1])):
        got.append([torch.zeros((n, 1, 128), dtype=torch.float16, device=DEV) for _ in range(2)])
        tkv.tkv_quantize_rows(desc, K, V, bits, None, *got[-1])
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(*got))


def test_tokens_far_into_a_packed_batch():
    n, hq, hk = 300000, 64, 1
    desc = tkv.tkv_desc.make(hk, 0, 0)
    q = torch.empty((n, hq, 128), dtype=torch.bfloat16, device=DEV)      # 4.9 GB
    q[-70:] = torch.randn((70, hq, 128), device=DEV).to(torch.bfloat16)
    k, v = (torch.randn((n, hk, 128), device=DEV).to(torch.bfloat16) for _ in range(2))
    out = torch.zeros((n, hq, 128), dtype=torch.bfloat16, device=DEV)
    plan = plan_of(128, 1 << 20, [n - 70, 70], [0, 0], hq // hk)
    plan = plan._replace(items=plan.items[plan.items[:, 0] == n - 70])
    prefill(desc, q, k, v, [None, None], plan, out)
    ref = torch.zeros((70, hq, 128), dtype=torch.bfloat16, device=DEV)
    prefill(desc, q[-70:], k[-70:], v[-70:], [None, None], plan_of(128, 1 << 20, [70], [0], hq // hk), ref)
    assert torch.equal(out[-70:], ref) and (out[:-70] == 0).all()


def test_rows_beyond_four_gigabytes():
    n, h = 1 << 20, 17
    desc = tkv.tkv_desc.make(h, 0, 0, int2_key_axis=1)
    K = torch.zeros((n, h, 128), dtype=torch.bfloat16, device=DEV)
    K[-200:] = torch.randn((200, h, 128), device=DEV).to(torch.bfloat16)
    bits = torch.zeros(n, dtype=torch.uint8, device=DEV)
    bits[-200:-100], bits[-96:-32], bits[-32:] = 4, 2, 4
    blocks = torch.arange(n - 96, n - 32, dtype=torch.int32, device=DEV)
    out = [torch.full((n, h, 128), 7.0, dtype=torch.float16, device=DEV) for _ in range(2)]
    tkv.tkv_quantize_rows(desc, K, K, bits, blocks, *out)
    ref = [torch.zeros((200, h, 128), dtype=torch.float16, device=DEV) for _ in range(2)]
    tkv.tkv_quantize_rows(desc, K[-200:], K[-200:], bits[-200:].clone(), blocks - (n - 200), *ref)
    torch.cuda.synchronize()
    for o, r in zip(out, ref):
        assert torch.equal(o[-200:], r) and (o[:-200] == 0).all()


@pytest.mark.parametrize("kind,n", [(torch.bfloat16, 150000), (torch.float32, 70000)])
def test_distortion_beyond_four_gigabytes(kind, n):
    h = 128
    x = torch.zeros((n, h, 128), dtype=kind, device=DEV)
    y = torch.zeros((n, h, 128), dtype=kind, device=DEV)
    x[-500:] = torch.randn((500, h, 128), device=DEV).to(kind)
    y[n // 2] = 1.0

    def call(x, y, ip):
        out = torch.zeros((len(ip) - 1, h), dtype=torch.float64, device=DEV)
        ws = torch.empty(tkv.tkv_distortion_workspace_bytes(len(ip) - 1, x.shape[0], h), dtype=torch.uint8, device=DEV)
        tkv.tkv_head_distortion(x, y, torch.tensor(ip, dtype=torch.int32, device=DEV), out, ws)
        torch.cuda.synchronize()
        return out

    got = call(x, y, [0, n // 2, n // 2 + 1, n - 500, n])
    want = (x[-500:].double() - y[-500:].double()).square().mean((0, 2))
    assert (got[0] == 0).all() and (got[1] == 1).all() and (got[2] == 0).all()
    assert ((got[3] - want).abs() <= (500 * 128 + 4) * 2.0 ** -52 * want).all()
