"""tkv_prefill_attention against attention in 64 bits (tests/prefill_model.py says where the tolerances come from)."""
import math

import numpy as np
import pytest
import torch

from paper_2605_17170_amd import tkv
from tests.prefill_model import attention, plan_of

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
SM = 1.0 / math.sqrt(128.0)
BF, FP = torch.bfloat16, torch.float16


def indptr(lens):
    return np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)


class Case:
    def __init__(self, lens, cached, hq, hk, q=BF, kv=BF, out=BF, packed=False, pad=0, spare=0, seed=0, target=256, sm=SM, size=1.0, kind=None, most=1 << 20):
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        self.lens, self.cached, self.hq, self.hk, self.sm = list(lens), list(cached), hq, hk, sm
        n, heads = sum(lens) + spare, hq + 2 * hk
        rows = torch.randn((n, heads * 128 + pad), device=DEV, generator=g)
        loud = torch.where(torch.rand((heads * 128 + pad,), device=DEV, generator=g) < 0.03, 10.0, 1.0)
        loud[:hq * 128] = size
        if packed:
            assert q == kv
            rows = (rows * loud).to(q)[:, :heads * 128].unflatten(1, (heads, 128))
            self.q, self.k, self.v = rows[:, :hq], rows[:, hq:hq + hk], rows[:, hq + hk:]
        else:
            rows = (rows * loud)[:, :heads * 128].unflatten(1, (heads, 128))
            self.q, self.k, self.v = rows[:, :hq].to(q).contiguous(), rows[:, hq:hq + hk].to(kv).contiguous(), rows[:, hq + hk:].to(kv).contiguous()
        m = sum(cached)
        self.before = [(torch.randn((m, hk, 128), device=DEV, generator=g) * 2.0).to(FP) if m else None for _ in range(2)]
        self.desc = tkv.tkv_desc.make(hk, 0, 0)
        self.plan = tkv.tkv_plan_prefill(self.desc, hq, indptr(lens), indptr(cached), target) if kind is None else plan_of(kind, most, lens, cached, hq // hk)
        self.prefill = tkv.tkv_prefill.make(self.plan, DEV)
        self.out = torch.full((n, hq, 128), 7.0, dtype=out, device=DEV)
        self.workspace = torch.full((max(16, tkv.tkv_prefill_workspace_bytes(self.desc, self.plan.n_slots, self.plan.tile_rows)),), 255, dtype=torch.uint8, device=DEV)
        self.status = torch.zeros(1, dtype=torch.int32, device=DEV)

    def call(self, **kw):
        return tkv.tkv_prefill_attention(self.desc, self.q, self.k, self.v, *self.before, self.prefill, self.sm, self.out, self.workspace, self.status, **kw)

    def check(self, what=""):
        torch.cuda.synchronize()
        assert int(self.status.item()) == 0
        ref, tol = attention(self.q, self.k, self.v, self.before, self.lens, self.cached, self.sm, self.out.dtype)
        n = sum(self.lens)
        got = self.out[:n].double()
        assert torch.isfinite(got).all(), what + ": not finite"
        off = (got - ref[:n]).abs() / tol[:n]
        worst = float(off.max()) if off.numel() else 0.0
        print("  %s: %.3f of the tolerance, %d slots" % (what, worst, self.plan.n_slots), flush=True)
        assert worst <= 1.0, "%s: %.3f of the tolerance at %s" % (what, worst, np.unravel_index(int(off.argmax()), off.shape))
        assert (self.out[n:] == 7.0).all(), "rows behind the last sequence"


TYPES = [(BF, BF, BF), (BF, FP, BF), (FP, FP, FP), (BF, BF, FP), (FP, FP, BF)]


@pytest.mark.parametrize("lens,cached,hq,hk", [
    ([1], [0], 1, 1), ([1], [1], 4, 1), ([2], [0], 8, 1), ([3, 1, 2], [0, 64, 5], 2, 2), ([63], [0], 1, 1), ([64], [63], 2, 1), ([65], [65], 4, 2),
    ([127, 0, 1], [0, 7, 0], 8, 8), ([129], [128], 1, 1), ([257, 31], [0, 1], 3, 1), ([200], [129], 10, 2), ([17, 300, 5], [500, 0, 77], 16, 1),
    ([33], [4001], 8, 2), ([1, 1, 1, 1], [1000, 1, 64, 129], 64, 8),
])
@pytest.mark.parametrize("types", TYPES)
def test_lengths_heads_and_types(lens, cached, hq, hk, types):
    c = Case(lens, cached, hq, hk, *types, spare=3, seed=len(lens) * 100 + hq)
    c.call()
    c.check("%s behind %s, %d on %d heads" % (lens, cached, hq, hk))


@pytest.mark.parametrize("pad", [0, 8, 72])
@pytest.mark.parametrize("kind", [BF, FP])
def test_parts_of_a_packed_projection(kind, pad):
    c = Case([70, 1, 130], [0, 33, 90], 8, 2, kind, kind, kind, packed=True, pad=pad, spare=5, seed=pad)
    c.call()
    c.check("packed, pad %d" % pad)


@pytest.mark.parametrize("rows", [32, 128, 256])
@pytest.mark.parametrize("most", [1, 2, 3, 7, 1 << 20])
@pytest.mark.parametrize("kv", [BF, FP])
def test_workgroups_of_every_kind_and_ranges_of_every_length(rows, most, kv):
    c = Case([5, 90, 1, 300], [1500, 70, 129, 0], 8, 2, BF, kv, BF, kind=rows, most=most, seed=rows + most % 100)
    assert (c.plan.n_slots > 0) == (most < 1000)
    c.call()
    c.check("%d rows, ranges of %d" % (rows, most))


@pytest.mark.parametrize("rows", [32, 128, 256])
@pytest.mark.parametrize("n", [1, 31, 32, 33, 63, 64, 65, 96, 127, 128, 129, 255, 256, 257, 383])
def test_one_head_at_the_borders_of_tiles(rows, n):
    for cached, most in ((0, 1 << 20), (n, 2)):
        c = Case([n], [cached], 1, 1, kind=rows, most=most, seed=n)
        c.call()
        c.check("%d rows, %d behind %d" % (rows, n, cached))


@pytest.mark.parametrize("parts", [31, 32, 33, 64, 70])
def test_many_parts(parts):
    c = Case([3], [32 * parts - 3], 4, 1, kind=32, most=1, seed=parts)
    assert c.plan.n_slots == parts + 0 + (1 if (32 * parts - 3) % 32 else 0)
    c.call()
    c.check("%d parts" % parts)


@pytest.mark.parametrize("target", [1, 3, 16, 256, 1024])
def test_plans_for_fewer_and_more_compute_units(target):
    c = Case([5, 90, 1], [3000, 700, 1500], 8, 2, target=target, seed=target)
    c.call()
    c.check("target %d, %d rows" % (target, c.plan.tile_rows))


def test_the_same_call_gives_the_same_bits():
    c = Case([150, 9], [2000, 64], 8, 2, seed=5)
    c.call()
    first = c.out.clone()
    for _ in range(3):
        c.out.fill_(7.0)
        c.workspace.fill_(255)
        c.call()
        assert torch.equal(c.out, first)


@pytest.mark.parametrize("rows", [32, 128, 256])
def test_a_sequence_does_not_depend_on_the_batch(rows):
    """With workgroups of one kind and whole ranges (which the plan chooses by the batch)."""
    c = Case([64, 100], [130, 0], 4, 2, seed=6, kind=rows)
    c.call()
    d = Case([100], [0], 4, 2, seed=7, kind=rows)
    d.q, d.k, d.v = c.q[64:].contiguous(), c.k[64:].contiguous(), c.v[64:].contiguous()
    d.call()
    assert torch.equal(c.out[64:], d.out)


@pytest.mark.parametrize("size,sm", [(40.0, SM), (1e-3, SM), (2.0 ** -110, SM * 2.0 ** 110), (2.0 ** 60, SM * 2.0 ** -60), (2.0 ** -122, 2.0 ** 118), (0.0, SM),
                                     (0.0, 2.0 ** -90), (1.0, 2.0 ** -100), (2.0 ** -120, 2.0 ** -20), (2.0 ** 120, 2.0 ** -126), (2.0 ** 100, 2.0 ** -120)])
@pytest.mark.parametrize("kv", [BF, FP])
def test_sizes_of_queries(size, sm, kv):
    c = Case([40], [100], 2, 1, BF, kv, BF, seed=8, sm=sm, size=size)
    c.call()
    c.check("size %g" % size)


def test_logits_far_apart_follow_the_maximum():
    c = Case([300], [64], 1, 1, seed=9)
    c.k[:] *= torch.linspace(0.1, 30.0, 300, device=DEV)[:, None, None].to(BF)      # the maximum keeps growing
    c.call()
    c.check("growing logits")


@pytest.mark.parametrize("kind", [BF, FP])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("rows,most", [(32, 3), (32, 1 << 20), (128, 2), (128, 1 << 20), (256, 1 << 20)])
def test_what_a_token_does_not_see_does_not_reach_it(kind, bad, rows, most):
    """NaN and infinities in keys and values of later tokens, of other sequences, of rows behind the last one."""
    lens, cached = [90, 70, 3], [70, 0, 1100]
    c = Case(lens, cached, 2, 1, kind, kind, kind, spare=4, seed=10, kind=rows, most=most)
    clean = Case(lens, cached, 2, 1, kind, kind, kind, spare=4, seed=10, kind=rows, most=most)
    clean.call()
    hit = [40, 90 + 69, 160 + 1]      # a token of each sequence
    for t in hit:
        c.k[t, 0, 5] = bad
        c.v[t, 0, 9] = bad
    c.k[163:], c.v[163:], c.q[163:] = bad, bad, bad
    c.call()
    torch.cuda.synchronize()
    before = torch.cat([torch.arange(0, 40), torch.arange(90, 159), torch.arange(160, 161)]).to(DEV)
    assert torch.equal(c.out[before], clean.out[before])
    assert (c.out[163:] == 7.0).all()


@pytest.mark.parametrize("kind", [BF, FP])
@pytest.mark.parametrize("at", [0, 63, 100, 149])
@pytest.mark.parametrize("rows", [32, 128, 256])
def test_values_that_are_not_finite_reach_the_tokens_that_see_them(kind, at, rows):
    c = Case([150], [0], 2, 1, kind, kind, kind, seed=11, kind=rows)
    clean = Case([150], [0], 2, 1, kind, kind, kind, seed=11, kind=rows)
    clean.call()
    c.v[at, 0, 3], c.v[at, 0, 40], c.v[at, 0, 127] = math.inf, -math.inf, math.nan
    c.call()
    torch.cuda.synchronize()
    assert (c.out[at:, :, 3] == math.inf).all() and (c.out[at:, :, 40] == -math.inf).all() and torch.isnan(c.out[at:, :, 127]).all()
    rest = [i for i in range(128) if i not in (3, 40, 127)]
    assert torch.equal(c.out[:at], clean.out[:at]) and torch.equal(c.out[:, :, rest], clean.out[:, :, rest])


def test_values_that_are_not_finite_in_prefixes_stay_in_their_sequence():
    c = Case([20, 30], [70, 100], 2, 1, seed=12, target=1)
    clean = Case([20, 30], [70, 100], 2, 1, seed=12, target=1)
    clean.call()
    c.before[1][3, 0, 7] = math.inf
    c.before[0][5, 0, 7] = math.nan
    c.call()
    torch.cuda.synchronize()
    assert torch.isnan(c.out[:20]).all() and torch.equal(c.out[20:], clean.out[20:])


@pytest.mark.parametrize("kv", [BF, FP])
@pytest.mark.parametrize("bad", [math.inf, math.nan])
def test_a_row_of_queries_that_is_not_finite_leaves_the_others_alone(kv, bad):
    c, clean = (Case([90], [40], 4, 2, BF, kv, BF, seed=13) for _ in range(2))
    clean.call()
    c.q[50, 2, 17] = bad
    c.call()
    torch.cuda.synchronize()
    assert torch.isnan(c.out[50, 2]).all()
    rest = torch.ones((90, 4), dtype=torch.bool, device=DEV)
    rest[50, 2] = False
    assert torch.equal(c.out[rest], clean.out[rest])


def test_on_another_stream_than_the_current_one():
    c = Case([100, 40], [300, 0], 8, 2, seed=14)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    c.call(stream=s)
    s.synchronize()
    c.check("other stream")


def test_two_calls_at_once_with_workspaces_of_their_own():
    a, b = Case([7], [5000], 8, 2, seed=15, kind=32, most=9), Case([9], [4000], 8, 2, seed=16, kind=128, most=9)
    assert a.plan.n_slots and b.plan.n_slots
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(5):
        a.call(stream=streams[0])
        b.call(stream=streams[1])
    for s in streams:
        s.synchronize()
    a.check("first")
    b.check("second")


def test_captured_and_replayed_with_other_inputs():
    c = Case([60, 1], [2000, 700], 8, 2, seed=17, kind=128, most=9)
    c.call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.call()
    for k in range(4):
        d = Case([60, 1], [2000, 700], 8, 2, seed=18 + k, kind=128, most=9)
        for x, y in zip([c.q, c.k, c.v] + c.before, [d.q, d.k, d.v] + d.before):
            x.copy_(y)
        c.out.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        d.call()
        torch.cuda.synchronize()
        assert torch.equal(c.out, d.out)
        c.check("replay %d" % k)


def test_two_captured_graphs_share_a_workspace():
    cases = [Case([60, 1], [2000, 700], 8, 2, seed=23, kind=128, most=9), Case([3], [6000], 8, 2, FP, FP, FP, seed=24, kind=32, most=5)]
    shared = max((c.workspace for c in cases), key=lambda w: w.numel())
    graphs = []
    for c in cases:
        assert c.plan.n_slots > 0
        c.workspace = shared
        c.call()
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            c.call()
    for k in (0, 1, 1, 0, 1, 0):
        cases[k].out.fill_(7.0)
        graphs[k].replay()
        cases[1 - k].call()
        graphs[k].replay()
        torch.cuda.synchronize()
        cases[0].check("replay")
        cases[1].check("replay")


@pytest.mark.parametrize("lens,cached,hq,hk", [([9, 2], [100, 0], 64, 1), ([3], [130], 300, 1), ([20, 70], [0, 65], 21, 3), ([40], [33], 32, 32), ([2, 5], [1, 900], 77, 7)])
@pytest.mark.parametrize("rows,most", [(32, 1 << 20), (128, 3), (256, 1 << 20)])
def test_groups_beyond_a_tile_and_of_odd_sizes(lens, cached, hq, hk, rows, most):
    c = Case(lens, cached, hq, hk, kind=rows, most=most, spare=2, seed=hq)
    c.call()
    c.check("%d on %d heads, %d rows" % (hq, hk, rows))


@pytest.mark.parametrize("rows,tokens", [(32, 1), (32, 31), (128, 3), (128, 128), (256, 200), (256, 256)])
@pytest.mark.parametrize("parts", [8, 9, 12, 17, 25, 40])
def test_parts_of_one_tile_of_every_kind(rows, tokens, parts):
    keys = 32 if rows == 32 else 64
    c = Case([tokens], [keys * parts], 1, 1, kind=rows, most=1, seed=parts, spare=1)
    assert c.plan.n_cut == 1 and c.plan.n_slots == parts + -(-tokens // keys)
    c.call()
    c.check("%d parts of %d rows" % (parts, rows))


def test_two_hundred_short_sequences():
    lens = [(7 * k) % 5 for k in range(200)]
    c = Case(lens, [(31 * k) % 190 for k in range(200)], 8, 2, seed=25, spare=4)
    c.call()
    c.check("200 sequences")


@pytest.mark.parametrize("word,value", [(0, -1), (0, 1000), (1, 0), (1, 1 << 30), (2, -1), (2, 1 << 30), (3, -1), (3, 1 << 20), (4, -128), (4, 1 << 30), (5, -1), (5, 99),
                                        (7, 1000), (7, -2), (8, -1), (8, 99), (9, 0), (9, 1 << 30)])
def test_items_that_name_what_is_not_there_are_skipped(word, value):
    c = Case([30, 20], [700, 3000], 4, 2, seed=19, kind=128, most=9)
    plan = c.plan._replace(items=c.plan.items.copy())
    first = int(np.flatnonzero(plan.items[:, 0] == 30)[0])
    plan.items[first, word] = value
    c.prefill = tkv.tkv_prefill.make(plan, DEV)
    c.call()
    torch.cuda.synchronize()
    assert int(c.status.item()) == tkv.TKV_STATUS_BAD_ITEM
    assert torch.isfinite(c.out[:30].float()).all()


@pytest.mark.parametrize("word,value", [(10, -1), (10, 40), (11, 0), (11, 60), (12, -8), (13, -1), (13, 1000), (14, 0), (14, 1000), (14, -3)])
def test_cut_tiles_that_name_what_is_not_there_are_skipped(word, value):
    c = Case([30, 20], [700, 3000], 4, 2, seed=19, kind=128, most=9)
    plan = c.plan._replace(items=c.plan.items.copy())
    assert plan.n_cut == 2 and plan.items[1, 10] == 30
    plan.items[1, word] = value
    c.prefill = tkv.tkv_prefill.make(plan, DEV)
    c.call()
    torch.cuda.synchronize()
    assert int(c.status.item()) == tkv.TKV_STATUS_BAD_ITEM
    assert torch.isfinite(c.out[:30].float()).all() and (c.out[30:] == 7.0).all()


def test_a_plan_without_items_and_a_call_without_tokens():
    c = Case([0, 0], [5, 0], 4, 2, spare=2)
    assert c.plan.items.shape == (0, 16) and c.plan.n_slots == 0
    c.call()
    torch.cuda.synchronize()
    assert (c.out == 7.0).all()
    tkv.tkv_prefill_attention(c.desc, c.q[:0], c.k[:0], c.v[:0], *c.before, c.prefill, SM, c.out[:0])
