"""tkv_decode_attention_shared at the ends of what its arguments may be, in items of 16, 64 and 128 rows."""
import numpy as np
import pytest
import torch

import gpu_common as gc
from paper_2605_17170_amd import harness, tkv
from paper_2605_17170_amd import workloads as wl
from test_gpu_shared import build, check, cut_rows, reference

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module", autouse=True)
def _oracle():
    from oracle import tkv_oracle
    tkv_oracle.build()


def attend(cache, q, sm_scale, workspace=None):
    """The batch of cache.plan_shared with another factor of the logits."""
    n, plan, prefix, d_items, d_indptr = cache._shared
    out = torch.empty(q.shape, dtype=torch.bfloat16, device=DEV)
    if workspace is None:
        workspace = torch.empty(tkv.tkv_decode_workspace_bytes(cache.desc, plan.n_slots, int(q.shape[1])), dtype=torch.uint8, device=DEV)
    tkv.tkv_decode_attention_shared(cache.desc, cache.pool, cache.bit_map, q, cache.d_page_indptr[n:], cache.d_page_ids, cache.d_n_tok2[n:], cache.d_n_tok4[n:],
                                    d_items, prefix, d_indptr, plan.n_slots, float(sm_scale), out, workspace, cache.status)
    torch.cuda.synchronize()
    assert int(cache.status.item()) == 0
    return out


def times(q, factor):
    """bf16 bits of q times a power of two, which is exact."""
    f = wl.bf16_bits_to_f32(q).astype(np.float32) * np.float32(factor)
    assert np.all(np.isfinite(f)) and not np.any(f.view(np.uint32) & 0xffff)
    return harness.bf16_tensor((f.view(np.uint32) >> 16).astype(np.uint16), DEV)


@pytest.mark.parametrize("key_axis", [0, 1])
def test_queries_from_the_smallest_to_the_largest_exponent(key_axis):
    """q times 2^k with a factor of the logits 2^-k as large: the same logits, and the same bits of the result."""
    cache, _, _ = build(71, [700], [30, 0, 130], 2, key_axis)
    try:
        q = wl.make_q(np.random.SeedSequence([71, 5]), 3, 16)
        f = np.clip(wl.bf16_bits_to_f32(q), -3.875, 3.875).astype(np.float32)
        f = np.where(np.abs(f) < 2.0 ** -12, 0.0, f).astype(np.float32)     # (the rest stays clear of subnormal numbers)
        f[2, 3] = 0.0
        q = (f.view(np.uint32) >> 16).astype(np.uint16)
        assert np.abs(f).max() >= 2.0
        cache.plan_shared([[0, 1, 2]], 16, 8, 8)
        scale = 16.0 * float(np.float32(gc.SM))     # (2^-126 of it is a normal number)
        for rows in (16, 64, 128):
            cut_rows(cache, rows, [3 * 8])
            want = attend(cache, times(q, 1.0), scale)
            assert torch.isfinite(want.float()).all()
            for k in (40, 100, 110, 116, 118, 122, 126, -40, -100, -114):
                got = attend(cache, times(q, 2.0 ** k), np.float32(scale) * np.float32(2.0 ** -k))
                assert torch.equal(got, want), (rows, k)
    finally:
        cache.close()


@pytest.mark.parametrize("key_axis", [0, 1])
def test_logits_too_small_for_32_bits_weigh_all_tokens_alike(key_axis):
    """A factor of the logits below the smallest number of 32 bits: the mean of the values, of these tokens only."""
    cache, Ks, Vs = build(73, [333], [20, 0, 65], 2, key_axis)
    try:
        q = wl.make_q(np.random.SeedSequence([73, 5]), 3, 8)
        cache.plan_shared([[0, 1, 2]], 8, 8, 8)
        want = reference(np.zeros_like(q), Ks, Vs, [[0, 1, 2]], 2)
        for rows in (16, 64, 128):
            cut_rows(cache, rows, [3 * 4])
            for k, scale in ((-100, 2.0 ** -70), (-60, 2.0 ** -126), (0, 1e-45)):
                f = wl.bf16_bits_to_f32(q).astype(np.float32) * np.float32(2.0 ** k)
                check(attend(cache, harness.bf16_tensor((f.view(np.uint32) >> 16).astype(np.uint16), DEV), scale), want, "%d rows, 2^%d, %g" % (rows, k, scale))
    finally:
        cache.close()


@pytest.mark.parametrize("key_axis", [0, 1])
@pytest.mark.parametrize("r", [2, 8])
def test_a_head_does_not_depend_on_what_the_others_ask(r, key_axis):
    """Other heads and sequences with other queries, small and huge ones and NaN: the same bits for those that stay."""
    cache, _, _ = build(83, [1500], [130, 0, 40, 64, 9], 2, key_axis)
    try:
        heads = 2 * r
        q = wl.make_q(np.random.SeedSequence([83, 5]), 5, heads)
        other = wl.make_q(np.random.SeedSequence([84, 5]), 5, heads)
        stay = np.random.default_rng(83).random((5, heads)) < 0.5
        cache.plan_shared([[0, 1, 2, 4]], heads, 8, 8)
        for rows in (16, 64, 128):
            cut_rows(cache, rows, [4 * r])
            want = attend(cache, harness.bf16_tensor(q, DEV), gc.SM)
            for factor in (1.0, 2.0 ** -20, 2.0 ** 9, 2.0 ** 30, float("nan")):
                f = np.where(stay[..., None], wl.bf16_bits_to_f32(q), wl.bf16_bits_to_f32(other) * np.float32(factor)).astype(np.float32)
                got = attend(cache, harness.bf16_tensor((f.view(np.uint32) >> 16).astype(np.uint16), DEV), gc.SM)
                mask = torch.from_numpy(stay).to(DEV)
                assert torch.equal(got[mask], want[mask]), (rows, factor)
    finally:
        cache.close()


@pytest.mark.parametrize("key_axis", [0, 1])
def test_a_head_whose_logits_are_all_infinite_is_nan(key_axis):
    """An infinity at a channel where all keys have one sign: every logit +inf or -inf, over a prefix alone, own tokens alone and both."""
    prefixes, own, kv_heads, r = [400], [30, 0, 0], 2, 4
    _, K, V, bits = gc.random_case(79, prefixes + own, kv_heads, kv_heads, f4=0.4)
    f = wl.bf16_bits_to_f32(K).astype(np.float32)
    f[..., 5] = 128.0 + np.abs(f[..., 5])     # the largest of its group of channels
    K = (f.view(np.uint32) >> 16).astype(np.uint16)
    cache = harness.PagedCache(kv_heads, bits, DEV, pool_factor=1.3, shuffle_seed=3, fill=0xFF, key_axis=key_axis)
    try:
        gc.gpu_append(cache, K, V)
        q = wl.make_q(np.random.SeedSequence([79, 5]), 3, kv_heads * r)
        bad = q.copy()
        where = [(0, 1, 0xff80), (0, 6, 0x7f80), (1, 2, 0xff80), (1, 3, 0x7f80), (1, 4, 0x7fc0), (2, 7, 0xffc1)]
        for b, h, bits_ in where:
            bad[b, h, 5] = bits_
        same = torch.ones((3, kv_heads * r), dtype=torch.bool, device=DEV)
        for b, h, _ in where:
            same[b, h] = False
        for groups in ([[0, 1]], [[1]]):      # (sequence 2 has no tokens at all: zeros, whatever q holds)
            cache.plan_shared(groups, kv_heads * r, 8, 8)
            for rows in (16, 64, 128):
                cut_rows(cache, rows, [len(groups[0]) * r])
                clean, out = (attend(cache, harness.bf16_tensor(x, DEV), gc.SM) for x in (q, bad))
                assert torch.isnan(out[:2][~same[:2]]).all(), (groups, rows)
                assert torch.equal(out[same], clean[same]) and bool((out[2] == 0).all()), (groups, rows)
    finally:
        cache.close()


@pytest.mark.parametrize("kv_heads,r,own", [(1, 1, [70, 0, 5]), (3, 1, [70, 20, 5]), (1, 8, [64, 0, 0]), (2, 4, [0, 0, 0]), (3, 8, [200, 1, 65])])
def test_partials_are_rows_of_512_bytes_behind_one_another(kv_heads, r, own):
    """acc of slot s and query head h at row s * heads + h of the workspace, (m, l) of all of them behind: merged here in 64 bits,
    off by the rounding to bf16, half a step of the result, and of the 32-bit sums."""
    heads = kv_heads * r
    cache, _, _ = build(89, [700], own, kv_heads)
    try:
        q = harness.bf16_tensor(wl.make_q(np.random.SeedSequence([89, 5]), 3, heads), DEV)
        plan = cache.plan_shared([[0, 2, 1]], heads, 3, 4)
        indptr = plan.seq_item_indptr.reshape(2, 4)
        for rows in (16, 64, 128):
            cut_rows(cache, rows, [3 * r])
            ws = torch.full((tkv.tkv_decode_workspace_bytes(cache.desc, plan.n_slots, heads) // 4,), float("nan"), device=DEV)
            out = attend(cache, q, gc.SM, ws).double().cpu()
            assert torch.isfinite(ws).all()
            n = plan.n_slots * heads
            acc, ml = ws[:128 * n].view(plan.n_slots, heads, 128).double().cpu(), ws[128 * n:].view(plan.n_slots, heads, 2).double().cpu()
            for b in range(3):
                at = [s for k in range(2) for s in range(indptr[k, b], indptr[k, b + 1])]
                w = torch.exp2(ml[at, :, 0] - ml[at, :, 0].amax(0))[..., None]
                den = (w[..., 0] * ml[at, :, 1]).sum(0)[:, None]
                want, size = (w * acc[at]).sum(0) / den, (w * acc[at].abs()).sum(0) / den
                assert bool(((out[b] - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -18 * size).all()), (rows, b)
    finally:
        cache.close()


@pytest.mark.parametrize("rows", [16, 64])
def test_more_workgroups_than_a_dimension_of_the_grid(rows):
    """2^23 + 5 parts, all but the last few of them empty: the same bits as the plan's parts by themselves in their slots."""
    cache, _, _ = build(97, [190], [70, 0], 1)
    try:
        q = harness.bf16_tensor(wl.make_q(np.random.SeedSequence([97, 5]), 2, 2), DEV)
        plan = cache.plan_shared([[1]], 2, 1, 1)
        cut_rows(cache, rows, [2])
        want = attend(cache, q, gc.SM)
        n, _, prefix, d_items, d_indptr = cache._shared
        old, n_own = prefix.tensors[7], d_items.shape[0]
        n_old, n_items = old.shape[0], (1 << 23) + 5
        items = torch.zeros((n_items, 5), dtype=torch.int32, device=DEV)      # (pages [0, 0) of group 0)
        items[:, 3] = torch.arange(n_items, dtype=torch.int32, device=DEV)
        items[-n_old:, [0, 1, 2, 4]] = old[:, [0, 1, 2, 4]]
        slots = torch.full((1,), n_own, dtype=torch.int32, device=DEV)
        indptr = d_indptr.clone()
        indptr[3:] = torch.tensor([n_own, n_own, n_own + n_items], dtype=torch.int32, device=DEV)
        many = tkv.tkv_prefix(1, 1, rows, n_items, *[t.data_ptr() for t in prefix.tensors[:6]], slots.data_ptr(), items.data_ptr())
        n_slots = n_own + n_items
        ws = torch.empty(tkv.tkv_decode_workspace_bytes(cache.desc, n_slots, 2), dtype=torch.uint8, device=DEV)
        out = torch.empty_like(want)
        tkv.tkv_decode_attention_shared(cache.desc, cache.pool, cache.bit_map, q, cache.d_page_indptr[n:], cache.d_page_ids, cache.d_n_tok2[n:],
                                        cache.d_n_tok4[n:], d_items, many, indptr, n_slots, gc.SM, out, ws, cache.status)
        torch.cuda.synchronize()
        assert int(cache.status.item()) == 0 and torch.isfinite(out.float()).all()
        assert torch.equal(out[0], want[0])
        # (the merge adds the same partials in another order: 32-bit sums, then half a step of bf16 on either side)
        assert bool(((out[1] - want[1]).float().abs() <= 2.0 ** -7 * want[1].float().abs() + 2.0 ** -16).all())
    finally:
        cache.close()


@pytest.mark.parametrize("key_axis", [0, 1])
def test_queries_that_are_subnormal_numbers(key_axis):
    """Multiples of 2^-133, the smallest bf16 number, up to fifteen of them, as the same multiples of 1/4."""
    cache, _, _ = build(103, [700], [30, 0, 130], 2, key_axis)
    try:
        f = np.clip(np.round(4 * wl.bf16_bits_to_f32(wl.make_q(np.random.SeedSequence([103, 5]), 3, 16))), -15, 15).astype(np.float32) / 4
        f[1] = np.clip(f[1], -0.25, 0.25)        # (all of these heads' values are subnormal then)
        q = (f.view(np.uint32) >> 16).astype(np.uint16)
        small = np.where(f < 0, 0x8000, 0).astype(np.uint16) | (4 * np.abs(f)).astype(np.uint16)     # (the bits of a subnormal number are its multiple)
        cache.plan_shared([[0, 1, 2]], 16, 8, 8)
        scale = np.float32(gc.SM) / np.float32(16)
        for rows in (16, 64, 128):
            cut_rows(cache, rows, [3 * 8])
            want = attend(cache, times(q, 1.0), scale)
            got = attend(cache, harness.bf16_tensor(small, DEV), scale * np.float32(2.0 ** 127) * np.float32(2.0 ** 4))
            assert torch.isfinite(want.float()).all() and torch.equal(got, want), rows
    finally:
        cache.close()
