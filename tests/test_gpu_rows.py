"""tkv_quantize_rows against the oracle's quantiser and its fp16 rows (bit for bit), and against append followed by gather."""
import numpy as np
import pytest
import torch

from oracle import tkv_oracle as orc
from paper_2605_17170_amd import harness, tkv
from paper_2605_17170_amd import workloads as wl

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def rows(seed, n, heads):
    K, V, _ = wl.make_kv(np.random.SeedSequence([seed, 3]), n, heads)
    return K, V


def widths(seed, lens, choices, channel_keys):
    """Widths of the tokens of each sequence in runs, and the blocks of per-channel keys."""
    rng = np.random.default_rng([seed, 5])
    out = []
    for n in lens:
        b = np.repeat(rng.choice(choices, n // 5 + 1), rng.integers(1, 40, n // 5 + 1))[:n].astype(np.uint8)
        b = np.concatenate([b, np.full(n - b.size, choices[0], np.uint8)])
        out.append(orc.route_residual(b) if channel_keys else b)
    return out


def blocks_of(seq_bits):
    base, out = 0, []
    for b in seq_bits:
        out.append(orc.int2_blocks(b, base))
        base += b.size
    return np.concatenate(out).astype(np.int64) if out else np.zeros((0, 32), np.int64)


def want(K, V, bits, blocks, channel_keys):
    """fp16 bit patterns."""
    res = []
    for part, x in enumerate((K, V)):
        codes, scale, zero = orc.quantize(x, np.where(bits == 0, 4, bits).astype(np.uint8))
        y = orc.dequantize_f16(codes, scale, zero)
        plain = orc.f32_to_f16(orc.bf16_to_f32(x).astype(np.float32)).reshape(x.shape)
        y[bits == 0] = plain[bits == 0]
        if part == 0 and channel_keys and blocks.size:
            bs, bz = orc.quantize_k_channel(x, blocks, codes)
            exact = np.zeros(x.shape, np.float64)
            orc.dequantize_k_channel(codes, blocks, bs, bz, exact)
            at = blocks.reshape(-1)
            y[at] = orc.f64_to_f16(exact[at]).reshape(y[at].shape)
        res.append(y)
    return res


def call(K, V, bits, blocks, channel_keys, packed=False, fill=7.0, expect=0):
    heads = K.shape[1]
    dK, dV = harness.bf16_tensor(K, DEV), harness.bf16_tensor(V, DEV)
    if packed:
        both = torch.cat([dK, dK, dV, dV[:, :, :8].repeat(1, 1, 16)], 1).contiguous()
        dK, dV = both[:, heads:2 * heads], both[:, 2 * heads:3 * heads]
    out = [torch.full(K.shape, fill, dtype=torch.float16, device=DEV) for _ in range(2)]
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    desc = tkv.tkv_desc.make(heads, 0, 0, int2_key_axis=1 if channel_keys else 0)
    dB = torch.from_numpy(np.ascontiguousarray(blocks, np.int32)).to(DEV) if channel_keys else None
    tkv.tkv_quantize_rows(desc, dK, dV, torch.from_numpy(bits).to(DEV), dB, *out, status)
    torch.cuda.synchronize()
    assert int(status.item()) == expect
    return [o.view(torch.int16).cpu().numpy().view(np.uint16) for o in out]


@pytest.mark.parametrize("lens,heads", [([1], 1), ([3], 2), ([31, 1], 5), ([64], 8), ([33, 500, 97], 4), ([1000], 1)])
@pytest.mark.parametrize("choices", [[0, 2], [0, 4], [2, 4], [0, 2, 4], [0], [2], [4]])
@pytest.mark.parametrize("channel_keys", [False, True])
def test_rows_equal_the_oracles(lens, heads, choices, channel_keys):
    seed = sum(lens) + heads
    K, V = rows(seed, sum(lens), heads)
    seq_bits = widths(seed, lens, choices, channel_keys)
    bits, blocks = np.concatenate(seq_bits), blocks_of(seq_bits) if channel_keys else np.zeros((0, 32), np.int64)
    if channel_keys:
        assert np.array_equal(tkv.tkv_plan_row_blocks(bits, np.concatenate([[0], np.cumsum(lens)])), blocks)
    for packed in (False, True):
        for got, ref in zip(call(K, V, bits, blocks, channel_keys, packed), want(K, V, bits, blocks, channel_keys)):
            assert np.array_equal(got, ref)


@pytest.mark.parametrize("channel_keys", [False, True])
def test_equal_to_append_and_gather(channel_keys):
    lens = [200, 65, 700]
    K, V = rows(3, sum(lens), 2)
    seq_bits = widths(4, lens, [2, 4], channel_keys)
    cache = harness.PagedCache(2, seq_bits, DEV, pool_factor=1.5, shuffle_seed=3, fill=0xA5, key_axis=1 if channel_keys else 0)
    try:
        cache.append(harness.bf16_tensor(K, DEV), harness.bf16_tensor(V, DEV))
        gathered = [torch.zeros(K.shape, dtype=torch.float16, device=DEV) for _ in range(2)]
        cache.gather(*gathered)
        torch.cuda.synchronize()
        assert int(cache.status.item()) == 0
        bits = np.concatenate(seq_bits)
        blocks = tkv.tkv_plan_row_blocks(bits, np.concatenate([[0], np.cumsum(lens)])) if channel_keys else None
        for got, ref in zip(call(K, V, bits, blocks, channel_keys), gathered):
            assert np.array_equal(got, ref.view(torch.int16).cpu().numpy().view(np.uint16))
    finally:
        cache.close()


def test_special_groups():
    """Constant groups, zeros of either sign, the smallest numbers, ranges whose scale is subnormal or zero, ties between codes."""
    x = np.zeros((12, 1, 128), np.float32)
    x[0] = -0.0
    x[1] = 3.25
    x[2, 0, ::2] = -0.0
    x[3] = np.linspace(0, 15, 128).astype(np.float32)
    x[4, 0, 5] = 1e-38
    x[5, 0, :] = np.arange(128) % 32 * 2.0 ** -24
    x[6] = np.where(np.arange(128) % 2, 65504.0, -65504.0)
    x[7, 0] = np.arange(128) % 31 / 2.0
    x[8, 0] = -np.abs(np.sin(np.arange(128)))
    x[9] = -1.0
    x[10, 0, 3] = -65000.0
    x[11, 0] = (np.arange(128) % 7) * 0.5
    K = (torch.from_numpy(x).to(torch.bfloat16).view(torch.int16).numpy().view(np.uint16)).reshape(12, 1, 128)
    for b in (0, 2, 4):
        bits = np.full(12, b, np.uint8)
        for got, ref in zip(call(K, K, bits, None, False), want(K, K, bits, np.zeros((0, 32)), False)):
            value, wanted = got.view(np.float16).astype(np.float64), ref.view(np.float16).astype(np.float64)
            assert np.array_equal(value, wanted)      # the sign of a zero is not the group's


def test_rows_left_alone_may_hold_anything():
    x = torch.randn((40, 2, 128), device=DEV).to(torch.bfloat16)
    x[3, 0, 5], x[3, 1, 6], x[4, 0, 7], x[5, 0, 1] = float("inf"), float("-inf"), float("nan"), 1e30
    bits = torch.full((40,), 4, dtype=torch.uint8, device=DEV)
    bits[3:6] = 0
    out = [torch.zeros((40, 2, 128), dtype=torch.float16, device=DEV) for _ in range(2)]
    tkv.tkv_quantize_rows(tkv.tkv_desc.make(2, 0, 0), x, x, bits, None, *out)
    torch.cuda.synchronize()
    for o in out:
        assert torch.equal(o[3:6].view(torch.int16), x[3:6].to(torch.float16).view(torch.int16)) or torch.isnan(o[4, 0, 7])
        assert torch.isfinite(o[:3]).all() and torch.isfinite(o[6:]).all() and o[3, 0, 5] == float("inf") and o[5, 0, 1] == float("inf") and torch.isnan(o[4, 0, 7])


def test_widths_and_blocks_that_cannot_be_are_skipped():
    K, V = rows(8, 70, 2)
    bits = np.full(70, 2, np.uint8)
    bits[64:] = 0
    ref = want(K, V, bits, np.arange(64).reshape(2, 32), True)
    odd = bits.copy()
    odd[66] = 3
    got = call(K, V, odd, np.arange(64).reshape(2, 32), True, expect=tkv.TKV_STATUS_TAG_MISMATCH)
    seven = np.float16(7.0).view(np.uint16)
    assert (got[0][66] == seven).all() and (got[1][66] == seven).all()
    keep = np.arange(70) != 66
    assert all(np.array_equal(g[keep], r[keep]) for g, r in zip(got, ref))
    for token in (70, -1, 64):
        blocks = np.arange(64).reshape(2, 32)
        blocks[1, 7] = token
        got = call(K, V, bits, blocks, True, expect=tkv.TKV_STATUS_BLOCK_PARTIAL)
        assert np.array_equal(got[0][:32], ref[0][:32]) and (got[0][32:64] == seven).all() and np.array_equal(got[1], ref[1])
    got = call(K, V, bits, np.arange(32).reshape(1, 32), True)      # a key that no block names
    assert (got[0][32:64] == seven).all() and np.array_equal(got[0][:32], ref[0][:32])


def test_on_another_stream_and_captured():
    K, V = rows(9, 300, 4)
    bits = widths(9, [300], [0, 2, 4], False)[0]
    ref = want(K, V, bits, np.zeros((0, 32)), False)
    dK, dV, dB = harness.bf16_tensor(K, DEV), harness.bf16_tensor(V, DEV), torch.from_numpy(bits).to(DEV)
    out = [torch.zeros(K.shape, dtype=torch.float16, device=DEV) for _ in range(2)]
    desc = tkv.tkv_desc.make(4, 0, 0)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    tkv.tkv_quantize_rows(desc, dK, dV, dB, None, *out, stream=s)
    s.synchronize()
    assert all(np.array_equal(o.view(torch.int16).cpu().numpy().view(np.uint16), r) for o, r in zip(out, ref))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        tkv.tkv_quantize_rows(desc, dK, dV, dB, None, *out)
    for _ in range(3):
        for o in out:
            o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(np.array_equal(o.view(torch.int16).cpu().numpy().view(np.uint16), r) for o, r in zip(out, ref))


def test_every_scale_that_bf16_numbers_give():
    """Groups from zero to every positive bf16 number that fp16 holds: all quotients by 3 and 15 and all reciprocals that occur."""
    most = np.arange(1, 0x4780, dtype=np.uint16)       # up to 65280
    most = np.concatenate([most, most[:-most.size % 4 or None][:(-most.size) % 4]])
    rng = np.random.default_rng(5)
    part = rng.random((most.size, 32))
    part[:, 0], part[:, 1], part[:, 2:8] = 0.0, 1.0, np.arange(1, 7) / 6.0      # the middles between codes of 2 bits among them
    x = torch.from_numpy(orc.bf16_to_f32(most).astype(np.float64)[:, None] * part).to(torch.float32).to(torch.bfloat16)
    x[:, 1] = torch.from_numpy(most.view(np.int16)).view(torch.bfloat16)
    K = x.view(torch.int16).numpy().view(np.uint16).reshape(-1, 1, 128)
    for b in (2, 4):
        bits = np.full(K.shape[0], b, np.uint8)
        for got, ref in zip(call(K, K, bits, None, False), want(K, K, bits, np.zeros((0, 32)), False)):
            assert np.array_equal(got, ref)
