"""The three operators as calibration runs them: rows of one tag at one width, replay, distortion.

Tolerance: the two replays are off by at most t0 and t1 for each value (tests/prefill_model.py), so their difference by t0 + t1, and the root of a
mean square by at most the root of the mean of (t0 + t1)^2.  Largest over heads, mean over requests and sum over layers keep that bound for each part."""
import math

import numpy as np
import pytest
import torch

from oracle import tkv_oracle as orc
from paper_2605_17170_amd import calibrate, harness, tkv
from paper_2605_17170_amd import workloads as wl
from tests.prefill_model import attention
from tests.test_gpu_rows import want

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
SM = 1.0 / math.sqrt(128.0)


def capture(seed, lens, hq, hk):
    ss = np.random.SeedSequence([seed, 9]).spawn(2)
    K, V, _ = wl.make_kv(ss[0], sum(lens), hk)
    q = wl.make_q(ss[1], sum(lens), hq)
    return q, K, V


def tags_of(seed, n):
    rng = np.random.default_rng([seed, 11])
    return np.repeat(rng.choice([0, 5, 22, 44], n // 9 + 1), rng.integers(1, 60, n // 9 + 1))[:n].astype(np.uint8)


def as_rows(x):
    return torch.from_numpy(x.view(np.int16)).view(torch.float16).to(DEV)


@pytest.mark.parametrize("key_axis", [0, 1])
def test_distortions_against_64_bits(key_axis):
    lens, hq, hk = [150, 1, 90], 4, 2
    ip = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    q, K, V = capture(1, lens, hq, hk)
    tags = tags_of(1, sum(lens))
    dq, dK, dV = (harness.bf16_tensor(x, DEV) for x in (q, K, V))
    r = calibrate.Replay(ip, hq, hk, SM, DEV, key_axis)
    r.attention(dq, dK, dV, np.zeros(tags.size, np.uint8), r.plain)

    def exact(widths):
        blocks = np.concatenate([orc.int2_blocks(widths[a:b], a) for a, b in zip(ip[:-1], ip[1:])]).astype(np.int64) if key_axis else np.zeros((0, 32), np.int64)
        rows = want(K, V, widths, blocks, key_axis == 1)
        return attention(dq, as_rows(rows[0]), as_rows(rows[1]), [None, None], lens, [0] * len(lens), SM, torch.float16)

    o0, t0 = exact(np.zeros(tags.size, np.uint8))
    for tag in np.unique(tags):
        for bits in (2, 4):
            got = r.distortion(dq, dK, dV, tags, int(tag), bits).cpu()
            o1, t1 = exact(r.widths(tags, int(tag), bits))
            for b in range(len(lens)):
                at = slice(int(ip[b]), int(ip[b + 1]))
                ref = (o1[at] - o0[at]).square().mean((0, 2)).cpu()
                off = (t0[at] + t1[at]).square().mean((0, 2)).sqrt().cpu()
                assert ((got[b].sqrt() - ref.sqrt()).abs() <= off).all(), "tag %d at %d bits, request %d" % (tag, bits, b)
    torch.cuda.synchronize()
    assert int(r.status.item()) == 0


def test_tables_feed_the_allocation():
    lens, hq, hk = [200, 333], 4, 1
    ip = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    tags = tags_of(3, sum(lens))
    layers = [[harness.bf16_tensor(x, DEV) for x in capture(s, lens, hq, hk)] for s in (4, 5)]
    N, D2, D4 = calibrate.tag_distortions(layers, tags, ip, SM)
    D = np.zeros((2, 56))
    for q, K, V in layers:
        r = calibrate.Replay(ip, hq, hk, SM, DEV)
        r.attention(q, K, V, np.zeros(tags.size, np.uint8), r.plain)
        for tag in np.unique(tags):
            for row, bits in enumerate((2, 4)):
                D[row, tag] += float(r.distortion(q, K, V, tags, int(tag), bits).amax(1).mean())
    assert np.array_equal(D[0], D2) and np.array_equal(D[1], D4)
    there = np.isin(np.arange(56), np.unique(tags))
    assert (D2[there] > D4[there]).all() and (D4[there] > 0).all() and (D2[~there] == 0).all()
    per = np.stack([np.bincount(tags[a:b], minlength=56) for a, b in zip(ip[:-1], ip[1:])])
    assert N[0] == int(np.median(per[:, 0])) and (N[1:7] == per.sum(0)[1:7]).all() and N.shape == (56,)
    bits = tkv.tkv_allocate_bits_greedy(N, D2, D4, 2.8)
    assert set(bits) <= {2, 4} and sum(n * b for n, b in zip(N, bits)) <= 2.8 * N.sum() * (1 + 2.0 ** -40)


def test_a_replay_captured_and_repeated():
    """One graph of the three calls; the widths change between replays, and eager work stands between them."""
    lens, hq, hk = [300, 77], 8, 2
    ip = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    q, K, V = (harness.bf16_tensor(x, DEV) for x in capture(6, lens, hq, hk))
    tags = tags_of(6, sum(lens))
    r = calibrate.Replay(ip, hq, hk, SM, DEV)
    r.attention(q, K, V, np.zeros(tags.size, np.uint8), r.plain)
    want_ = {(t, b): r.distortion(q, K, V, tags, t, b).clone() for t in np.unique(tags).tolist() for b in (2, 4)}
    bits = torch.zeros(tags.size, dtype=torch.uint8, device=DEV)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        tkv.tkv_quantize_rows(r.desc, K, V, bits, None, r.K, r.V, r.status)
        tkv.tkv_prefill_attention(r.desc, q, r.K, r.V, None, None, r.prefill, SM, r.out, r.workspace, r.status)
        tkv.tkv_head_distortion(r.plain, r.out, r.d_indptr, r.by_head, r.sums)
    for (t, b), ref in want_.items():
        bits.copy_(torch.from_numpy(r.widths(tags, t, b)))
        r.by_head.fill_(-1.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(r.by_head, ref), (t, b)
        r.out.zero_()
    assert int(r.status.item()) == 0


@pytest.mark.parametrize("key_axis", [0, 1])
def test_prompts_behind_a_cached_prefix(key_axis):
    """As a serving loop runs them: old tokens in the paged cache, gathered to fp16 rows; new ones normed, rotated, appended and attended to."""
    hq, hk, old, new = 8, 2, [200, 64, 333], [40, 130, 1]
    rng = np.random.default_rng(13)
    bits = [np.repeat(rng.choice([2, 4], n // 7 + 1), 7)[:n].astype(np.uint8) for n in old]
    K, V, _ = wl.make_kv(np.random.SeedSequence([14, 3]), sum(old), hk)
    cache = harness.PagedCache(hk, bits, DEV, pool_factor=2.0, shuffle_seed=5, fill=0xA5, key_axis=key_axis)
    try:
        cache.append(harness.bf16_tensor(K, DEV), harness.bf16_tensor(V, DEV))
        before = [torch.zeros((sum(old), hk, 128), dtype=torch.float16, device=DEV) for _ in range(2)]
        cache.gather(*before)
        g = torch.Generator(device=DEV)
        g.manual_seed(15)
        rows = torch.randn((sum(new), hq + 2 * hk, 128), device=DEV, generator=g).to(torch.bfloat16)
        q, k, v = rows[:, :hq], rows[:, hq:hq + hk], rows[:, hq + hk:]
        turned = [torch.empty(x.shape, dtype=torch.bfloat16, device=DEV) for x in (q, k)]
        positions = torch.cat([torch.arange(a, a + n) for a, n in zip(old, new)]).to(torch.int32).to(DEV)[None].contiguous()
        weight = torch.ones(128, device=DEV).to(torch.bfloat16)
        tkv.tkv_norm_rope(tkv.tkv_rope_make(128, device=DEV), q, k, None, positions, weight, weight, 1e-6, *turned)
        ip = lambda n: np.concatenate([[0], np.cumsum(n)]).astype(np.int32)  # noqa: E731
        plan = tkv.tkv_plan_prefill(cache.desc, hq, ip(new), ip(old), harness.default_shared_units())
        out = torch.zeros((sum(new), hq, 128), dtype=torch.bfloat16, device=DEV)
        ws = torch.empty(max(16, tkv.tkv_prefill_workspace_bytes(cache.desc, plan.n_slots, plan.tile_rows)), dtype=torch.uint8, device=DEV)
        tkv.tkv_prefill_attention(cache.desc, turned[0], turned[1], v, *before, tkv.tkv_prefill.make(plan, DEV), SM, out, ws, cache.status)
        torch.cuda.synchronize()
        assert int(cache.status.item()) == 0
        ref, tol = attention(turned[0], turned[1], v, before, new, old, SM, torch.bfloat16)
        assert ((out.double() - ref).abs() <= tol).all()
    finally:
        cache.close()
