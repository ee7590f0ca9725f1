"""Plan of shared prefixes, and the refusals of tkv_decode_attention_shared that need no GPU: nothing here launches anything."""
import ctypes as C

import numpy as np
import pytest

from paper_2605_17170_amd import tkv

DESC = tkv.tkv_desc.make(4, 1000, 1000)


def plan(batch, heads, n2, n4, groups, target, n_own=0, desc=DESC):
    indptr = np.concatenate([[0], np.cumsum([len(g) for g in groups])])
    sip = np.minimum(np.arange(batch + 1), n_own)
    sip[-1] = n_own
    return tkv.tkv_plan_decode_shared(desc, batch, heads, n2, n4, indptr, [b for g in groups for b in g], target, np.zeros((n_own, 4), np.int32), sip)


@pytest.mark.parametrize("seed", range(40))
def test_items_cover_the_pages_and_slots_are_the_sequences(seed):
    rng = np.random.default_rng(seed)
    batch, n, r = int(rng.integers(1, 30)), int(rng.integers(0, 5)), int(rng.choice([1, 2, 4, 8]))
    groups = [rng.permutation(batch)[:rng.integers(0, batch + 1)].tolist() for _ in range(n)]
    n2, n4 = rng.integers(0, 9000, n) * (rng.random(n) < 0.7), rng.integers(0, 9000, n) * (rng.random(n) < 0.7)
    target, n_own = int(rng.integers(1, 400)), int(rng.integers(0, 9))
    p = plan(batch, 4 * r, n2, n4, groups, target, n_own)
    pages = -(-n2 // 64) + -(-n4 // 64)
    tile = p.max_members.tile_rows
    assert tile in (16, 64, 128)
    unit, per_group = 8 if tile == 16 else 2, []
    launched, split = 0, []
    for g in range(n):
        items = p.prefix_items[p.prefix_items[:, 0] == g]
        launched += len(items) * 4
        blocks = -(-len(groups[g]) * r // tile)
        if blocks:
            assert np.array_equal(items[:, 4], np.tile(np.arange(blocks) * tile, len(items) // blocks))     # every row of every part
            items = items.reshape(-1, blocks, 5)
            assert np.all(items[:, :, :4] == items[:, :1, :4])
            items = items[:, 0]
        per_group.append(len(items))
        if not groups[g] or pages[g] == 0:
            assert len(items) == 0
            continue
        assert items[0, 1] == 0 and items[-1, 2] == pages[g] and np.array_equal(items[1:, 1], items[:-1, 2]) and np.all(items[:, 2] > items[:, 1])
        assert np.array_equal(items[:, 3], np.arange(len(items)))
        wide = -(-n2[g] // 64)      # first page of the second width
        split.append(not np.any((items[:, 1] < wide) & (items[:, 2] > wide)) and 0 < wide < pages[g])
        for part in [items[items[:, 1] < wide], items[items[:, 1] >= wide]] if split[-1] else [items]:
            units = -(-(part[:, 2] - part[:, 1]) // unit)
            assert units.max() - units.min() <= 1 and np.all((part[:-1, 2] - part[0, 1]) % unit == 0)
    fewest = sum(4 * -(-len(groups[g]) * r // tile) for g in range(n) if per_group[g])
    assert launched <= max(target, fewest)
    # slots of a sequence: one of each item of each of its groups, all different, side by side, behind the own ones
    indptr = p.seq_item_indptr[batch + 1:]
    assert indptr[0] == n_own and indptr[-1] == p.n_slots and p.max_members == max([len(g) for g in groups], default=0)
    taken = [set() for _ in range(batch)]
    at = 0
    for g in range(n):
        for b in groups[g]:
            for k in range(per_group[g]):
                slot = int(p.member_slots[at]) + k
                assert slot not in taken[b]
                taken[b].add(slot)
            at += 1
    for b in range(batch):
        assert taken[b] == set(range(indptr[b], indptr[b + 1]))


def raw(**kw):
    a = dict(desc=DESC, batch=3, heads=8, n=1, n2=[100], n4=[100], indptr=[0, 2], seqs=[0, 2], target=4, own=0, cap=100)
    a.update(kw)
    arr = lambda x: np.array(x, np.int32) if x is not None else None  # noqa: E731
    ptr = lambda x: C.c_void_p(x.ctypes.data) if x is not None and x.size else None  # noqa: E731
    n2, n4, ip, sq = (arr(a[k]) for k in ("n2", "n4", "indptr", "seqs"))
    items, slots, out, tile = np.empty((max(1, a["cap"]), 5), np.int32), np.empty(16, np.int32), np.empty(64, np.int32), C.c_int32(0)
    return tkv.lib().tkv_plan_decode_shared(C.byref(a["desc"]), a["batch"], a["heads"], a["n"], ptr(n2), ptr(n4), ptr(ip), ptr(sq), a["target"], a["own"],
                                            ptr(items), a["cap"], ptr(slots), ptr(out), C.byref(tile))


@pytest.mark.parametrize("kw,status", [
    (dict(desc=tkv.tkv_desc.make(0, 1, 1)), tkv.TKV_ERR_BAD_SHAPE), (dict(batch=-1), tkv.TKV_ERR_INVALID_ARG), (dict(n=-1), tkv.TKV_ERR_INVALID_ARG),
    (dict(heads=0), tkv.TKV_ERR_INVALID_ARG), (dict(heads=6), tkv.TKV_ERR_BAD_SHAPE), (dict(heads=12), tkv.TKV_ERR_BAD_SHAPE), (dict(heads=64), tkv.TKV_ERR_BAD_SHAPE),
    (dict(target=0), tkv.TKV_ERR_INVALID_ARG), (dict(target=(1 << 31) - 1), tkv.TKV_ERR_INVALID_ARG), (dict(own=-1), tkv.TKV_ERR_INVALID_ARG),
    (dict(n2=[-1]), tkv.TKV_ERR_INVALID_ARG), (dict(n4=None), tkv.TKV_ERR_INVALID_ARG), (dict(indptr=[1, 2]), tkv.TKV_ERR_INVALID_ARG),
    (dict(indptr=[0, -1]), tkv.TKV_ERR_INVALID_ARG), (dict(seqs=[0, 3]), tkv.TKV_ERR_INVALID_ARG), (dict(seqs=[-1, 2]), tkv.TKV_ERR_INVALID_ARG),
    (dict(seqs=[2, 2]), tkv.TKV_ERR_INVALID_ARG),                                      # a sequence twice in a group would count the prefix twice
    (dict(seqs=None), tkv.TKV_ERR_INVALID_ARG), (dict(cap=0), tkv.TKV_ERR_CAPACITY),
    (dict(desc=tkv.tkv_desc.make(4, 10, 10, int2_key_axis=1)), tkv.TKV_ERR_INVALID_ARG),   # 100 INT2 tokens are no whole blocks
    (dict(n=0, n2=[], n4=[], indptr=[0], seqs=[]), 0), (dict(batch=0, indptr=[0, 0], seqs=[]), 0),
])
def test_plan_refusals(kw, status):
    assert raw(**kw) == status


def test_a_plan_of_hundreds_of_millions_of_tokens_does_not_overflow():
    d = tkv.tkv_desc.make(1, 2 ** 24, 2 ** 23)     # (two pools of 2^24 pages are more than a descriptor may name)
    p = plan(2, 1, [2 ** 31 - 1 - 63], [2 ** 31 - 1 - 63], [[0, 1]], 10, desc=d)
    assert p.prefix_items[-1, 2] == 2 * -(-(2 ** 31 - 64) // 64) and len(p.prefix_items) <= 30


def call(**kw):
    """tkv_decode_attention_shared with addresses that are never touched."""
    d = dict(n_groups=1, n_members=2, tile_rows=64, n_items=1, page_indptr=64, page_ids=64, n_tok_int2=64, n_tok_int4=64, member_indptr=64,
             member_seqs=64, member_slots=64, items=64)
    a = dict(desc=DESC, pool=256, bit_map=256, q=256, indptr=64, ids=64, n2=64, n4=64, items=64, n_items=3, slots=64, n_slots=9, batch=3, heads=8, scale=0.1,
             out=256, ws=256, ws_bytes=1 << 30, status=64)
    for k, v in kw.items():
        (d if k in d and k not in ("items", "n_items") else a)[k.replace("p_", "")] = v
    for k in ("p_items", "p_n_items"):
        if k in kw:
            d[k[2:]] = kw[k]
            a[k[2:]] = 64 if k == "p_items" else 3
    prefix = tkv.tkv_prefix(*(d[f] for f, _ in tkv.tkv_prefix._fields_)) if kw.get("prefix", 1) is not None else None
    by = lambda x: C.byref(x) if x is not None else None  # noqa: E731
    return tkv.lib().tkv_decode_attention_shared(by(a["desc"]), a["pool"], a["bit_map"], a["q"], a["indptr"], a["ids"], a["n2"], a["n4"], a["items"], a["n_items"],
                                                 by(prefix), a["slots"], a["n_slots"], a["batch"], a["heads"], a["scale"], a["out"], a["ws"], a["ws_bytes"],
                                                 a["status"], None)


BAD = tkv.TKV_ERR_INVALID_ARG


@pytest.mark.parametrize("kw,status", [
    (dict(prefix=None), BAD), (dict(desc=None), BAD), (dict(desc=tkv.tkv_desc.make(4, 1, 1, head_dim=64)), tkv.TKV_ERR_BAD_SHAPE),
    (dict(heads=6), tkv.TKV_ERR_BAD_SHAPE), (dict(heads=64), tkv.TKV_ERR_BAD_SHAPE), (dict(n_items=-1), BAD), (dict(n_slots=2), BAD), (dict(batch=-1), BAD),
    (dict(ws_bytes=9 * 8 * 130 * 4 - 1), tkv.TKV_ERR_WORKSPACE_TOO_SMALL), (dict(ws=None), BAD), (dict(ws=264), BAD),
    (dict(scale=0.0), BAD), (dict(scale=float("nan")), BAD), (dict(q=None), BAD), (dict(q=264), BAD), (dict(out=None), BAD), (dict(out=264), BAD),
    (dict(slots=None), BAD), (dict(pool=None), BAD), (dict(pool=128), BAD), (dict(bit_map=None), BAD), (dict(indptr=None), BAD), (dict(ids=None), BAD),
    (dict(items=None), BAD), (dict(n2=None), BAD),
    (dict(n_groups=-1), BAD), (dict(n_groups=0), BAD), (dict(n_members=0), BAD),
    (dict(p_n_items=-1), BAD), (dict(p_n_items=1 << 29), BAD), (dict(p_items=None), BAD), (dict(page_indptr=None), BAD), (dict(page_ids=None), BAD),
    (dict(n_tok_int2=None), BAD), (dict(n_tok_int4=None), BAD), (dict(member_indptr=None), BAD), (dict(member_seqs=None), BAD), (dict(member_slots=None), BAD),
    (dict(tile_rows=0), BAD), (dict(tile_rows=32), BAD), (dict(n_members=1 << 30), BAD),
    (dict(batch=0), tkv.TKV_OK),
])
def test_calls_that_launch_nothing(kw, status):
    assert call(**kw) == status


def test_a_prefix_wants_the_plan_s_own_number_of_members():
    import torch
    i32 = lambda n: torch.zeros(n, dtype=torch.int32)  # noqa: E731
    p = plan(2, 4, [100], [100], [[0, 1]], 10)
    prefix = tkv.tkv_prefix.make(i32(2), i32(4), i32(1), i32(1), i32(2), i32(2), i32(2), torch.from_numpy(p.prefix_items), p.max_members)
    assert prefix.n_items == len(p.prefix_items) and prefix.tile_rows == p.max_members.tile_rows
    with pytest.raises(ValueError):
        tkv.tkv_prefix.make(i32(2), i32(4), i32(1), i32(1), i32(2), i32(2), i32(2), torch.from_numpy(p.prefix_items), 2)
