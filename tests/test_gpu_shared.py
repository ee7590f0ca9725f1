"""tkv_decode_attention_shared against attention in 64 bits over the values that stand in the cache.

Tolerance.  With p the softmax weights and dl the largest error of a logit, a weighted mean of V is off by at most
(e^(2 dl) - 1) * sum p |V - out| <= 2.2 dl (sum p |V| + |out|).  K is rounded (not for own tokens and items of 16 rows) to fp16, half a step 2^-11 of each value: dl <=
scale * sum |q K| * 2^-11 (the 32-bit sums add 2^-17 of the same sum).  Weights and V are rounded to fp16: 2 * 2^-11 of sum p |V|,
the denominator by none of its own (it sums the rounded weights).  Then one rounding to bf16, 2^-8 of the result."""
import numpy as np
import pytest
import torch

import gpu_common as gc
from paper_2605_17170_amd import harness, tkv
from paper_2605_17170_amd import workloads as wl

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module", autouse=True)
def _oracle():
    from oracle import tkv_oracle
    tkv_oracle.build()


def build(seed, prefixes, own, kv_heads, key_axis=0, f4=0.4, fill=0xFF, shuffle_seed=3, k_exp=0):
    """A cache of prefix lists and own lists; (cache, K, V in 64 bits per list)."""
    _, K, V, bits = gc.random_case(seed, list(prefixes) + list(own), kv_heads, kv_heads, f4=f4)
    K = ((wl.bf16_bits_to_f32(K).astype(np.float32) * np.float32(2.0 ** k_exp)).view(np.uint32) >> 16).astype(np.uint16)
    cache = harness.PagedCache(kv_heads, bits, DEV, pool_factor=1.3, shuffle_seed=shuffle_seed, fill=fill, key_axis=key_axis)
    gc.gpu_append(cache, K, V)
    if key_axis:
        _, Kq, Vq, tok, bs, bz = gc.kc_oracle(bits, K, V)
        Kh, Vh = gc.kc_dequantized(Kq, Vq, tok, bs, bz)
    else:
        Kq, Vq = gc.orc.quantize(K, cache.tag_bits), gc.orc.quantize(V, cache.tag_bits)
        Kh, Vh = gc.orc.dequantize(*Kq), gc.orc.dequantize(*Vq)
    ends = np.cumsum([b.size for b in bits])[:-1]
    return cache, np.split(np.asarray(Kh, np.float64), ends), np.split(np.asarray(Vh, np.float64), ends)


def reference(q, Ks, Vs, groups, kv_heads, rounded=True):
    """(result, tolerance) [batch, heads, 128] in 64 bits; q bf16 bits.  rounded: keys are fp16 numbers, and a logit is off by half
    a step of each; otherwise by the 32-bit sums of (code - 1) s + (z + s), whose parts are at most three times the largest key of
    a group or of a channel's block, 2^-24 for each of 128 channels."""
    n, f = len(groups), wl.bf16_bits_to_f32(q).astype(np.float64)
    batch, heads = f.shape[:2]
    r = heads // kv_heads
    out, tol = np.zeros(f.shape), np.zeros(f.shape)
    for b in range(batch):
        lists = [g for g in range(n) if b in groups[g]] + [n + b]
        K, V = (torch.from_numpy(np.concatenate([X[i] for i in lists]).transpose(1, 0, 2).copy()) for X in (Ks, Vs))
        if K.shape[1] == 0:
            continue
        x = torch.from_numpy(f[b].reshape(kv_heads, r, 128))
        logits = torch.matmul(x, K.transpose(1, 2).contiguous()) * gc.SM
        p = torch.softmax(logits, -1)
        o, size = torch.matmul(p, V), torch.matmul(p, V.abs())
        dl = (torch.matmul(x.abs(), K.abs().transpose(1, 2).contiguous()).amax(-1, keepdim=True) * gc.SM) * (2.0 ** -11 + 2.0 ** -17)
        if not rounded:
            big = torch.maximum(K.abs().reshape(kv_heads, -1, 4, 32).amax(-1, keepdim=True).expand(-1, -1, 4, 32).reshape(K.shape), K.abs().amax(1, keepdim=True))
            dl = 3.0 * 2.0 ** -17 * torch.matmul(x.abs(), big.transpose(1, 2).contiguous()).amax(-1, keepdim=True) * gc.SM
        t = 2.0 ** -8 * o.abs() + 2.2 * dl * (size + o.abs()) + 2.0 * 2.0 ** -11 * size + 1e-30
        out[b], tol[b] = o.reshape(heads, 128).numpy(), t.reshape(heads, 128).numpy()
    return out, tol


def check(out, want, what=""):
    got, (ref, tol) = out.float().cpu().numpy().astype(np.float64), want
    assert np.all(np.isfinite(got)), what
    worst = float((np.abs(got - ref) / np.maximum(tol, 1e-30)).max())
    rel = float(np.linalg.norm(got - ref) / max(np.linalg.norm(ref), 1e-300))
    print("  %s: %.3f of the tolerance, %.2e in norm" % (what, worst, rel), flush=True)
    assert worst <= 1.0, (what, worst)


def cut_rows(cache, rows, rows_of_group):
    """The plan's parts with items of another number of rows."""
    prefix = cache._shared[2]
    parts = np.unique(prefix.tensors[7].cpu().numpy().reshape(-1, 5)[:, :4], axis=0)
    items = np.array([[*p, row] for p in parts for row in range(0, rows_of_group[p[0]], rows)], np.int32).reshape(-1, 5)
    cache._shared = (*cache._shared[:2], tkv.tkv_prefix(prefix.n_groups, prefix.n_members, rows, len(items), *[t.data_ptr() for t in prefix.tensors[:7]], 0),
                     *cache._shared[3:])
    cache._shared[2].tensors = (*prefix.tensors[:7], torch.from_numpy(items).to(DEV))
    cache._shared[2].items = cache._shared[2].tensors[7].data_ptr()


def run(seed, prefixes, own, groups, kv_heads, r, key_axis=0, f4=0.4, target_items=40, target_cus=8, q=None, k_exp=0):
    cache, Ks, Vs = build(seed, prefixes, own, kv_heads, key_axis, f4, k_exp=k_exp)
    try:
        q = wl.make_q(np.random.SeedSequence([seed, 5]), len(own), kv_heads * r) if q is None else q
        cache.plan_shared(groups, kv_heads * r, target_items, target_cus)
        want = {exact: reference(q, Ks, Vs, groups, kv_heads, not exact) for exact in (False, True)}
        for rows in (16, 64, 128):     # the plan chooses one by the sizes; each has to hold at every size
            cut_rows(cache, rows, [len(g) * r for g in groups])
            out = cache.decode_shared(harness.bf16_tensor(q, DEV))
            torch.cuda.synchronize()
            assert int(cache.status.item()) == 0
            check(out, want[rows == 16], "%s %s in %d rows" % (prefixes, own, rows))
        return out
    finally:
        cache.close()


@pytest.mark.parametrize("key_axis", [0, 1])
@pytest.mark.parametrize("kv_heads,r", [(1, 1), (2, 2), (1, 4), (3, 8)])
@pytest.mark.parametrize("members", [1, 2, 5, 9, 20])
def test_heads_and_members(kv_heads, r, members, key_axis):
    own = [(7 * i + 3) % 90 for i in range(members)]
    run(members * 10 + r, [700], own, [list(range(members))], kv_heads, r, key_axis)


@pytest.mark.parametrize("key_axis", [0, 1])
@pytest.mark.parametrize("length", [1, 31, 32, 33, 63, 64, 65, 127, 255, 256, 257, 1000])
def test_lengths_of_the_prefix(length, key_axis):
    run(length, [length], [0, 1, 40], [[0, 1, 2]], 2, 4, key_axis)


@pytest.mark.parametrize("f4", [0.0, 1.0])
@pytest.mark.parametrize("key_axis", [0, 1])
def test_one_width_only(f4, key_axis):
    run(3, [517], [64, 5], [[0, 1]], 1, 8, key_axis, f4=f4)


def test_groups_that_nest_are_empty_or_have_no_tokens():
    # everything for all, a document for some, a group without members, a prefix without tokens, a sequence in none, one without any token
    run(11, [300, 130, 77, 0], [50, 0, 10, 64, 3, 0], [[0, 1, 2, 3], [3, 1], [], [2, 0]], 2, 4)


def test_no_prefix_at_all_and_nothing_of_their_own():
    run(13, [], [100, 0, 3], [], 2, 2)
    run(17, [200], [0, 0, 0], [[2, 0, 1]], 2, 2)
    run(19, [0], [0, 0], [[0, 1]], 1, 1)


@pytest.mark.parametrize("key_axis", [0, 1])
def test_long_items(key_axis):
    # one workgroup per head: more than 64 pages for each of its wavefronts, and pages of both widths on either side of a batch
    run(23, [20011], [5, 130], [[1, 0]], 1, 4, key_axis, f4=0.25, target_cus=1)
    run(29, [20011], [5, 130], [[1, 0]], 1, 4, key_axis, f4=0.6, target_cus=1)


@pytest.mark.parametrize("target_cus", [1, 3, 50, 1000])
def test_any_number_of_items_gives_the_same(target_cus):
    run(31, [1900, 650], [20, 30, 40, 50, 60], [[0, 2, 4], [1, 3]], 2, 8, target_cus=target_cus)


def test_queries_of_very_different_size():
    q = wl.bf16_bits_to_f32(wl.make_q(np.random.SeedSequence([37, 5]), 4, 8)).astype(np.float32)
    q[0] *= 2.0 ** 40          # a softmax that is all one token
    q[1] *= 2.0 ** -60
    q[2, 3] = 0.0
    q[3, :, ::2] *= 2.0 ** -14
    bits = (q.view(np.uint32) >> 16).astype(np.uint16)
    cache, Ks, Vs = build(37, [333], [20, 0, 64, 1], 2)
    try:
        cache.plan_shared([[0, 1, 2, 3]], 8, 8, 8)
        out = cache.decode_shared(harness.bf16_tensor(bits, DEV))
        torch.cuda.synchronize()
        assert int(cache.status.item()) == 0
        ref, tol = reference(bits, Ks, Vs, [[0, 1, 2, 3]], 2)
        check(out, (ref, tol), "scaled")
    finally:
        cache.close()


@pytest.mark.parametrize("key_axis", [0, 1])
@pytest.mark.parametrize("k_exp", [7, -12])
def test_keys_large_and_small(k_exp, key_axis):
    # up to 2^14, and with scales down to the smallest normal numbers and below
    q = wl.bf16_bits_to_f32(wl.make_q(np.random.SeedSequence([39, 5]), 3, 8)).astype(np.float32) * np.float32(2.0 ** -k_exp)
    run(39, [700], [100, 3, 70], [[0, 1, 2]], 2, 4, key_axis, q=(q.view(np.uint32) >> 16).astype(np.uint16), k_exp=k_exp)


def test_queries_beyond_fp16_over_a_prefix_alone():
    q = wl.bf16_bits_to_f32(wl.make_q(np.random.SeedSequence([38, 5]), 2, 8)).astype(np.float32)
    q[0] *= 2.0 ** 40
    run(38, [333], [0, 0], [[0, 1]], 2, 4, q=(q.view(np.uint32) >> 16).astype(np.uint16))


def test_a_query_head_of_nan_or_infinities_leaves_the_others():
    cache, Ks, Vs = build(41, [400], [30, 0, 70], 2)
    try:
        q = wl.make_q(np.random.SeedSequence([41, 5]), 3, 8)
        cache.plan_shared([[0, 1, 2]], 8, 8, 8)
        clean = cache.decode_shared(harness.bf16_tensor(q, DEV)).clone()
        bad = q.copy()
        bad[0, 1, 5], bad[1, 4, 0], bad[2, 7, 127] = 0x7fc0, 0x7f80, 0xff80     # NaN, inf, -inf
        out = cache.decode_shared(harness.bf16_tensor(bad, DEV))
        torch.cuda.synchronize()
        same = torch.ones((3, 8), dtype=torch.bool, device=DEV)
        for b, h in ((0, 1), (1, 4), (2, 7)):
            same[b, h] = False
            assert torch.isnan(out[b, h]).all(), (b, h)
        assert torch.equal(out[same], clean[same])
    finally:
        cache.close()


def test_pages_that_cannot_be_read_count_nothing():
    """Ids outside the pool or of the other width, pages never written: flagged, and left out."""
    n = 64 * 6
    cache, Ks, Vs = build(43, [n], [10, 20], 1, f4=1.0)
    try:
        q = wl.make_q(np.random.SeedSequence([43, 5]), 2, 4)
        cache.plan_shared([[0, 1]], 4, 4, 4)
        ids = cache.d_page_ids.clone()
        keep, bits = np.ones(n, bool), 0
        for page, value, bit in ((1, -1, tkv.TKV_STATUS_PAGE_RANGE), (2, 1 << 30, tkv.TKV_STATUS_PAGE_RANGE), (3, 0, tkv.TKV_STATUS_BITMAP_MISMATCH)):
            cache.status.zero_()
            cache.d_page_ids[page] = value
            cache.decode_shared(harness.bf16_tensor(q, DEV))
            torch.cuda.synchronize()
            bits |= bit       # the pages of the rounds before are still bad
            assert int(cache.status.item()) == bits, (page, value)
            keep[64 * page:64 * page + 64] = False
        cache.status.zero_()
        cache.bit_map[int(ids[4])] = 2
        keep[256:320] = False
        out = cache.decode_shared(harness.bf16_tensor(q, DEV))
        torch.cuda.synchronize()
        assert int(cache.status.item()) == tkv.TKV_STATUS_BITMAP_MISMATCH | tkv.TKV_STATUS_PAGE_RANGE
        check(out, reference(q, [Ks[0][keep]] + Ks[1:], [Vs[0][keep]] + Vs[1:], [[0, 1]], 1), "pages left out")
    finally:
        cache.close()


def test_members_slots_and_items_that_cannot_be():
    cache, Ks, Vs = build(47, [300], [10, 20, 30], 1)
    try:
        q = harness.bf16_tensor(wl.make_q(np.random.SeedSequence([47, 5]), 3, 4), DEV)
        plan = cache.plan_shared([[0, 1, 2]], 4, 4, 2)
        clean = cache.decode_shared(q).clone()
        n, _, prefix, _, _ = cache._shared
        seqs, slots, items = prefix.tensors[5], prefix.tensors[6], prefix.tensors[7]
        guard = 4096
        size = tkv.tkv_decode_workspace_bytes(cache.desc, plan.n_slots, 4)
        ws = torch.full((size + guard,), 0x11, dtype=torch.uint8, device=DEV)

        def flagged(t, at, value):
            old = t.reshape(-1)[at].clone()
            t.reshape(-1)[at] = value
            cache.status.zero_()
            out = cache.decode_shared(q, workspace=ws[:size])
            torch.cuda.synchronize()
            t.reshape(-1)[at] = old
            assert int(cache.status.item()) == tkv.TKV_STATUS_BAD_ITEM, (at, value)
            assert bool((ws[size:] == 0x11).all())
            return out

        for value in (-1, 3, 1 << 30, -(1 << 31)):
            assert torch.equal(flagged(seqs, 1, value)[[0, 2]], clean[[0, 2]])
        for value in (-1, plan.n_slots, (1 << 31) - 1, 0):
            assert torch.equal(flagged(slots, 1, value)[[0, 2]], clean[[0, 2]])
        flagged(items, 0, -1)
        flagged(items, 0, 1)
        flagged(items, 3, -1)
        flagged(items, 4, -1)
        flagged(items, 4, -(1 << 31))
        flagged(items, 3, (1 << 31) - 1)
    finally:
        cache.close()


def test_pages_beyond_offsets_of_32_bits():
    """The same cache with its pages 5 GiB into either arena of a larger pool."""
    kv_heads, heads = 2, 8
    cache, Ks, Vs = build(61, [900], [30, 130, 0], kv_heads)
    try:
        q = harness.bf16_tensor(wl.make_q(np.random.SeedSequence([61, 5]), 3, heads), DEV)
        plan = cache.plan_shared([[2, 0, 1]], heads, 8, 8)
        p2, p4 = cache.desc.n_pages_int2, cache.desc.n_pages_int4
        size2, size4 = (tkv.tkv_page_bytes(cache.desc, bits) for bits in (2, 4))
        far2, far4 = (5 << 30) // size2, (5 << 30) // size4
        desc = tkv.tkv_desc.make(kv_heads, p2 + far2, p4 + far4)
        pool = torch.empty(tkv.tkv_pool_bytes(desc), dtype=torch.uint8, device=DEV)
        bit_map = torch.zeros(p2 + far2 + p4 + far4, dtype=torch.uint8, device=DEV)
        for page, far, n, size in ((0, far2, p2, size2), (p2, far2 + far4, p4, size4)):
            a, b = tkv.tkv_record_offset(cache.desc, page, 0), tkv.tkv_record_offset(desc, page + far, 0)
            pool[b:b + n * size] = cache.pool[a:a + n * size]
            bit_map[page + far:page + far + n] = cache.bit_map[page:page + n]
        ids = torch.where(cache.d_page_ids < p2, cache.d_page_ids + far2, cache.d_page_ids + far2 + far4)
        assert tkv.tkv_record_offset(desc, int(ids.min()), 0) > 1 << 32
        out = torch.empty(q.shape, dtype=torch.bfloat16, device=DEV)
        ws = torch.empty(tkv.tkv_decode_workspace_bytes(desc, plan.n_slots, heads), dtype=torch.uint8, device=DEV)
        for rows in (16, 64, 128):
            cut_rows(cache, rows, [3 * heads // kv_heads])
            want = cache.decode_shared(q)
            _, _, near, d_items, d_indptr = cache._shared
            prefix = tkv.tkv_prefix(*[getattr(near, f) for f, _ in tkv.tkv_prefix._fields_])
            prefix.page_ids = ids.data_ptr()
            tkv.tkv_decode_attention_shared(desc, pool, bit_map, q, cache.d_page_indptr[1:], ids, cache.d_n_tok2[1:], cache.d_n_tok4[1:], d_items, prefix,
                                            d_indptr, plan.n_slots, float(gc.SM), out, ws, cache.status)
            torch.cuda.synchronize()
            assert int(cache.status.item()) == 0 and torch.equal(out, want), rows
    finally:
        cache.close()


def test_captured_and_replayed_with_other_queries_and_counts():
    cache, Ks, Vs = build(53, [640], [100, 40, 64], 2)
    try:
        q = harness.bf16_tensor(wl.make_q(np.random.SeedSequence([53, 5]), 3, 8), DEV)
        plan = cache.plan_shared([[0, 1, 2]], 8, 8, 8)
        out, eager = torch.empty(q.shape, dtype=torch.bfloat16, device=DEV), torch.empty(q.shape, dtype=torch.bfloat16, device=DEV)
        ws = [torch.empty(tkv.tkv_decode_workspace_bytes(cache.desc, plan.n_slots, 8), dtype=torch.uint8, device=DEV) for _ in range(2)]
        cache.decode_shared(q, out, ws[0])
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            cache.decode_shared(q, out, ws[0])
        for step in range(4):
            q.mul_(-1.5)
            cache.d_n_tok4[1:] -= 1       # shorter by a token each
            cache.decode_shared(q, eager, ws[1])
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, eager), step
        assert int(cache.status.item()) == 0
    finally:
        cache.close()


def test_on_another_stream_and_two_at_once():
    cache, Ks, Vs = build(59, [1500], [10, 20, 30, 40], 2)
    try:
        q = harness.bf16_tensor(wl.make_q(np.random.SeedSequence([59, 5]), 4, 8), DEV)
        cache.plan_shared([[0, 1, 3]], 8, 8, 8)
        want = cache.decode_shared(q).clone()
        torch.cuda.synchronize()
        streams, outs = [torch.cuda.Stream() for _ in range(2)], []
        for s in streams:
            with torch.cuda.stream(s):
                for _ in range(5):
                    outs.append(cache.decode_shared(q))
        torch.cuda.synchronize()
        assert all(torch.equal(o, want) for o in outs)
    finally:
        cache.close()
