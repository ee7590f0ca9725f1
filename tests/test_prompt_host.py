"""Plans of prompt attention and of per-channel blocks, and the refusals of tkv_prefill_attention, tkv_quantize_rows and tkv_head_distortion that
need no GPU: nothing here launches anything."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2605_17170_amd import tkv

KEYS = {32: 32, 128: 64, 256: 64}


def plan(lens, cached, hq, hk, target=256):
    ip = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    pp = None if cached is None else np.concatenate([[0], np.cumsum(cached)]).astype(np.int32)
    return tkv.tkv_plan_prefill(tkv.tkv_desc.make(hk, 0, 0), hq, ip, pp, target)


@pytest.mark.parametrize("lens,cached,hq,hk", [
    ([1], None, 1, 1), ([0, 0], [3, 0], 4, 2), ([5, 0, 700], [0, 9, 64], 8, 2), ([1] * 40, [1000] * 40, 64, 8), ([4000], [30000], 64, 8), ([3], [1000000], 8, 1),
    ([8192, 1, 77], [0, 5000, 63], 5, 5), ([129, 64, 65, 63], [64, 65, 63, 1], 12, 4), ([20000], None, 64, 8), ([1] * 3000, None, 7, 1), ([31, 33], [100000, 1], 3, 1),
])
@pytest.mark.parametrize("target", [1, 64, 256, 5000])
def test_every_row_meets_every_key_that_it_sees_once(lens, cached, hq, hk, target):
    p = plan(lens, cached, hq, hk, target)
    group, rows, keys = hq // hk, p.tile_rows, KEYS[p.tile_rows]
    cached = cached or [0] * len(lens)
    starts, pres = np.concatenate([[0], np.cumsum(lens)]), np.concatenate([[0], np.cumsum(cached)])
    want = {}
    for b, (n, c) in enumerate(zip(lens, cached)):
        for r in range(0, n * group, rows):
            see = (min(r + rows, n * group) - 1) // group + 1
            want[(b, r)] = -(-c // keys) + -(-see // keys)
    seen, slots, cuts = {}, [], []
    owner = {(int(starts[b]), int(lens[b])): b for b in range(len(lens)) if lens[b]}
    for it in p.items.tolist():
        token0, n, prefix0, c, row, begin, end, slot, part, parts = it[:10]
        b = owner[(token0, n)]
        assert c == cached[b] and (c == 0 or prefix0 == pres[b]) and begin < end
        ranges = seen.setdefault((b, row), [])
        assert part == len(ranges) and (ranges == [] and begin == 0 or ranges[-1][1] == begin)
        ranges.append((begin, end, parts, slot))
        if parts > 1:
            slots.append(slot)
            if part == 0:
                cuts.append([token0, n, row, slot, parts])
        else:
            assert slot == -1
    assert seen.keys() == want.keys()
    for at, ranges in seen.items():
        assert ranges[-1][1] == want[at] and all(r[2] == len(ranges) for r in ranges)
        if len(ranges) > 1:
            assert [r[3] for r in ranges] == list(range(ranges[0][3], ranges[0][3] + len(ranges)))
    assert sorted(slots) == list(range(p.n_slots)) and p.n_cut == len(cuts)
    assert p.items[:len(cuts), 10:15].tolist() == cuts and not p.items[len(cuts):, 10:15].any() and not p.items[:, 15].any()
    assert len(p.items) <= tkv.lib().tkv_plan_prefill_capacity(C.byref(tkv.tkv_desc.make(hk, 0, 0)), len(lens), sum(lens), hq, target)
    lengths = [r[-1][1] / len(r) for r in ([(x[0], x[1]) for x in v] for v in seen.values())]
    if p.tile_rows == 128 and not p.n_slots:      # the longest ones of a first round last
        first = max(1, target // hk)
        assert lengths[:first] == sorted(lengths[:first]) or len(lengths) <= first
        lengths = lengths[:first][::-1] + lengths[first:] if len(lengths) > first else lengths
    assert lengths == sorted(lengths, reverse=True)


def test_longer_batches_never_make_more_workgroups_than_twice_the_places_when_cut():
    for lens, cached, hq, hk in (([1], [200000], 8, 1), ([1] * 7, [30000] * 7, 64, 8), ([60, 5], [9000, 70000], 8, 2)):
        p = plan(lens, cached, hq, hk)
        assert p.n_slots and len(p.items) * hk <= 4 * 256 + hk


def raw_plan(desc, batch, hq, ip, pp, target=4, cap=100):
    items = np.zeros((max(cap, 1), 16), np.int32)
    out = [C.c_int32(-7) for _ in range(3)]
    keep = [None if a is None else np.ascontiguousarray(a, np.int32) for a in (ip, pp)]
    return tkv.lib().tkv_plan_prefill(C.byref(desc) if desc is not None else None, batch, hq, *(None if a is None else C.c_void_p(a.ctypes.data) for a in keep), target,
                                      C.c_void_p(items.ctypes.data), cap, *(C.byref(o) for o in out))


def test_plans_that_cannot_be():
    d = tkv.tkv_desc.make(2, 0, 0)
    assert raw_plan(d, 1, 4, [0, 5], None) > 0
    assert raw_plan(d, 0, 4, [0], None) == 0
    for args, status in [((None, 1, 4, [0, 5], None), tkv.TKV_ERR_INVALID_ARG), ((tkv.tkv_desc.make(0, 0, 0), 1, 4, [0, 5], None), tkv.TKV_ERR_BAD_SHAPE),
                         ((tkv.tkv_desc.make(2, 0, 0, head_dim=64), 1, 4, [0, 5], None), tkv.TKV_ERR_BAD_SHAPE), ((d, 1, 3, [0, 5], None), tkv.TKV_ERR_BAD_SHAPE),
                         ((d, 1, 0, [0, 5], None), tkv.TKV_ERR_INVALID_ARG), ((d, -1, 4, [0], None), tkv.TKV_ERR_INVALID_ARG), ((d, 1, 4, None, None), tkv.TKV_ERR_INVALID_ARG),
                         ((d, 1, 4, [1, 5], None), tkv.TKV_ERR_INVALID_ARG), ((d, 2, 4, [0, 5, 4], None), tkv.TKV_ERR_INVALID_ARG), ((d, 1, 4, [0, 5], [1, 2]), tkv.TKV_ERR_INVALID_ARG),
                         ((d, 2, 4, [0, 5, 6], [0, 5, 4]), tkv.TKV_ERR_INVALID_ARG), ((d, 1, 4, [0, 5], None, 0), tkv.TKV_ERR_INVALID_ARG),
                         ((d, 1, 4, [0, 5], None, 4, -1), tkv.TKV_ERR_INVALID_ARG), ((d, 2, 4, [0, 5, 9], None, 4, 1), tkv.TKV_ERR_CAPACITY),
                         ((d, 1, 1 << 20, [0, 1 << 20], None), tkv.TKV_ERR_INVALID_ARG)]:
        assert raw_plan(*args) == status, args
    with pytest.raises(ValueError):
        tkv.tkv_plan_prefill(d, 4, [0, 5], [0])
    L, c = tkv.lib(), lambda *a: tkv.lib().tkv_plan_prefill_capacity(C.byref(d), *a)  # noqa: E731
    assert c(-1, 5, 4, 1) == c(1, -5, 4, 1) == c(1, 5, 4, 0) == tkv.TKV_ERR_INVALID_ARG and c(1, 5, 3, 1) == tkv.TKV_ERR_BAD_SHAPE
    assert c(1, (1 << 31) - 1, 1 << 20, 1) == tkv.TKV_ERR_INVALID_ARG
    assert [L.tkv_prefill_workspace_bytes(C.byref(d), *a) for a in ((-1, 32), (3, 64), (3, 0), (0, 128))] == [0, 0, 0, 0]
    assert L.tkv_prefill_workspace_bytes(C.byref(d), 3, 128) == 3 * 2 * 128 * 130 * 4


def prefill_args(**kw):
    p = tkv.tkv_prefill(32, 1, 0, 0, 4096)
    a = dict(desc=C.byref(tkv.tkv_desc.make(2, 0, 0)), hq=4, q=4096, qs=512, qt=0, K=4096, ks=256, V=4096, vs=256, kt=0, n=3, kp=None, vp=None, np=0, prefill=p, sm=0.1,
             out=4096, ot=0, ws=None, wb=0, status=None, stream=None)
    a.update(kw)
    if a["prefill"] is not None:
        a["prefill"] = C.byref(a["prefill"])
    return list(a.values())


@pytest.mark.parametrize("kw,status", [
    (dict(desc=None), tkv.TKV_ERR_INVALID_ARG), (dict(hq=3), tkv.TKV_ERR_BAD_SHAPE), (dict(hq=0), tkv.TKV_ERR_INVALID_ARG), (dict(prefill=None), tkv.TKV_ERR_INVALID_ARG),
    (dict(n=-1), tkv.TKV_ERR_INVALID_ARG), (dict(np=-1), tkv.TKV_ERR_INVALID_ARG), (dict(prefill=tkv.tkv_prefill(32, -1, 0, 0, 4096)), tkv.TKV_ERR_INVALID_ARG),
    (dict(prefill=tkv.tkv_prefill(32, 1, -1, 0, 4096)), tkv.TKV_ERR_INVALID_ARG), (dict(prefill=tkv.tkv_prefill(32, 1, 0, -1, 4096)), tkv.TKV_ERR_INVALID_ARG),
    (dict(prefill=tkv.tkv_prefill(32, 1, 0, 1, 4096)), tkv.TKV_ERR_INVALID_ARG), (dict(prefill=tkv.tkv_prefill(64, 1, 0, 0, 4096)), tkv.TKV_ERR_INVALID_ARG),
    (dict(prefill=tkv.tkv_prefill(32, 1, 0, 0, None)), tkv.TKV_ERR_INVALID_ARG), (dict(prefill=tkv.tkv_prefill(32, 1, 0, 0, 4098)), tkv.TKV_ERR_INVALID_ARG),
    (dict(qt=2), tkv.TKV_ERR_INVALID_ARG), (dict(kt=2), tkv.TKV_ERR_INVALID_ARG), (dict(ot=2), tkv.TKV_ERR_INVALID_ARG), (dict(qt=1, kt=0), tkv.TKV_ERR_INVALID_ARG),
    (dict(qt=-1), tkv.TKV_ERR_INVALID_ARG), (dict(sm=0.0), tkv.TKV_ERR_INVALID_ARG), (dict(sm=-1.0), tkv.TKV_ERR_INVALID_ARG), (dict(sm=float("nan")), tkv.TKV_ERR_INVALID_ARG),
    (dict(sm=float("inf")), tkv.TKV_ERR_INVALID_ARG), (dict(q=None), tkv.TKV_ERR_INVALID_ARG), (dict(q=4104), tkv.TKV_ERR_INVALID_ARG), (dict(qs=511), tkv.TKV_ERR_INVALID_ARG),
    (dict(qs=504), tkv.TKV_ERR_INVALID_ARG), (dict(qs=-512), tkv.TKV_ERR_INVALID_ARG), (dict(ks=1 << 23), tkv.TKV_ERR_INVALID_ARG), (dict(K=None), tkv.TKV_ERR_INVALID_ARG),
    (dict(V=4100), tkv.TKV_ERR_INVALID_ARG), (dict(vs=248), tkv.TKV_ERR_INVALID_ARG), (dict(np=5), tkv.TKV_ERR_INVALID_ARG), (dict(np=5, kp=4096), tkv.TKV_ERR_INVALID_ARG),
    (dict(np=5, kp=4096, vp=4104), tkv.TKV_ERR_INVALID_ARG), (dict(out=None), tkv.TKV_ERR_INVALID_ARG), (dict(out=4100), tkv.TKV_ERR_INVALID_ARG),
    (dict(ws=4100), tkv.TKV_ERR_INVALID_ARG), (dict(status=4098), tkv.TKV_ERR_INVALID_ARG), (dict(prefill=tkv.tkv_prefill(32, 2, 2, 1, 4096)), tkv.TKV_ERR_INVALID_ARG),
    (dict(prefill=tkv.tkv_prefill(32, 2, 2, 1, 4096), ws=4096, wb=2 * 2 * 32 * 130 * 4 - 1), tkv.TKV_ERR_WORKSPACE_TOO_SMALL),
    (dict(prefill=tkv.tkv_prefill(32, 1 << 30, 0, 0, 4096)), tkv.TKV_ERR_INVALID_ARG),
])
def test_prompt_attention_refuses(kw, status):
    assert tkv.lib().tkv_prefill_attention(*prefill_args(**kw)) == status


def test_prompt_attention_without_work_is_nothing():
    assert tkv.lib().tkv_prefill_attention(*prefill_args(prefill=tkv.tkv_prefill(32, 0, 0, 0, None), q=None, K=None, V=None, out=None)) == tkv.TKV_OK
    assert tkv.lib().tkv_prefill_attention(*prefill_args(n=0, q=None, K=None, V=None, out=None)) == tkv.TKV_OK


@pytest.mark.parametrize("kw,status", [
    (dict(desc=None), tkv.TKV_ERR_INVALID_ARG), (dict(desc=C.byref(tkv.tkv_desc.make(2, 0, 0, group_size=64))), tkv.TKV_ERR_BAD_SHAPE), (dict(n=-1), tkv.TKV_ERR_INVALID_ARG),
    (dict(nb=-1), tkv.TKV_ERR_INVALID_ARG), (dict(nb=2, blocks=4096), tkv.TKV_ERR_INVALID_ARG), (dict(nb=1), tkv.TKV_ERR_INVALID_ARG), (dict(nb=1, blocks=4098), tkv.TKV_ERR_INVALID_ARG),
    (dict(desc=C.byref(tkv.tkv_desc.make(2, 0, 0)), nb=1, blocks=4096), tkv.TKV_ERR_INVALID_ARG), (dict(K=None), tkv.TKV_ERR_INVALID_ARG), (dict(V=4104), tkv.TKV_ERR_INVALID_ARG),
    (dict(ks=255), tkv.TKV_ERR_INVALID_ARG), (dict(vs=128), tkv.TKV_ERR_INVALID_ARG), (dict(bits=None), tkv.TKV_ERR_INVALID_ARG), (dict(ko=None), tkv.TKV_ERR_INVALID_ARG),
    (dict(vo=4104), tkv.TKV_ERR_INVALID_ARG), (dict(status=4097), tkv.TKV_ERR_INVALID_ARG), (dict(n=1 << 30), tkv.TKV_ERR_INVALID_ARG),
])
def test_rows_refuses(kw, status):
    a = dict(desc=C.byref(tkv.tkv_desc.make(2, 0, 0, int2_key_axis=1)), K=4096, ks=256, V=4096, vs=256, bits=4096, n=40, blocks=None, nb=0, ko=4096, vo=4096, status=None, stream=None)
    a.update(kw)
    assert tkv.lib().tkv_quantize_rows(*a.values()) == status


def test_rows_without_tokens_is_nothing():
    assert tkv.lib().tkv_quantize_rows(C.byref(tkv.tkv_desc.make(2, 0, 0)), None, 0, None, 0, None, 0, None, 0, None, None, None, None) == tkv.TKV_OK


@pytest.mark.parametrize("kw,status", [
    (dict(t=3), tkv.TKV_ERR_INVALID_ARG), (dict(t=-1), tkv.TKV_ERR_INVALID_ARG), (dict(b=-1), tkv.TKV_ERR_INVALID_ARG), (dict(n=-1), tkv.TKV_ERR_INVALID_ARG),
    (dict(h=-1), tkv.TKV_ERR_INVALID_ARG), (dict(ip=None), tkv.TKV_ERR_INVALID_ARG), (dict(ip=4098), tkv.TKV_ERR_INVALID_ARG), (dict(out=None), tkv.TKV_ERR_INVALID_ARG),
    (dict(out=4100), tkv.TKV_ERR_INVALID_ARG), (dict(x=None), tkv.TKV_ERR_INVALID_ARG), (dict(y=4104), tkv.TKV_ERR_INVALID_ARG), (dict(ws=None), tkv.TKV_ERR_INVALID_ARG),
    (dict(ws=4104), tkv.TKV_ERR_INVALID_ARG), (dict(wb=8), tkv.TKV_ERR_WORKSPACE_TOO_SMALL), (dict(n=1 << 30, h=4), tkv.TKV_ERR_INVALID_ARG),
])
def test_distortion_refuses(kw, status):
    a = dict(x=4096, y=4096, t=0, ip=4096, b=2, n=100, h=4, out=4096, ws=4096, wb=1 << 20, stream=None)
    a.update(kw)
    assert tkv.lib().tkv_head_distortion(*a.values()) == status


def test_distortion_of_nothing_is_nothing():
    assert tkv.lib().tkv_head_distortion(None, None, 0, None, 0, 5, 3, None, None, 0, None) == tkv.TKV_OK
    assert tkv.lib().tkv_head_distortion(None, None, 0, None, 3, 5, 0, None, None, 0, None) == tkv.TKV_OK
    assert tkv.tkv_distortion_workspace_bytes(-1, 5, 5) == tkv.tkv_distortion_workspace_bytes(1, -5, 5) == tkv.tkv_distortion_workspace_bytes(1, 5, -5) == 0


def test_blocks_of_every_sequence():
    bits = np.array([2] * 20 + [0] * 3 + [2] * 12 + [4] * 5 + [2] * 64, np.uint8)
    got = tkv.tkv_plan_row_blocks(bits, [0, 40, 40, 104])
    assert got.tolist() == [list(range(20)) + list(range(23, 35)), list(range(40, 72)), list(range(72, 104))]
    assert tkv.tkv_plan_row_blocks([], [0]).shape == (0, 32) and tkv.tkv_plan_row_blocks([4] * 70, [0, 70]).shape == (0, 32)
    with pytest.raises(tkv.TkvError):
        tkv.tkv_plan_row_blocks(bits, [0, 30, 104])
    with pytest.raises(ValueError):
        tkv.tkv_plan_row_blocks(bits, [0, 30])
    L = tkv.lib()
    b, ip, out = np.full(64, 2, np.uint8), np.array([0, 64], np.int32), np.zeros(64, np.int32)
    p = lambda a: C.c_void_p(a.ctypes.data)  # noqa: E731
    assert L.tkv_plan_row_blocks(p(b), p(ip), 1, p(out), 1) == tkv.TKV_ERR_CAPACITY and L.tkv_plan_row_blocks(p(b), p(ip), 1, p(out), 2) == 2
    bad = np.array([0, 64, 32], np.int32)
    for args in ((p(b), None, 1, p(out), 2), (None, p(ip), 1, p(out), 2), (p(b), p(ip), -1, p(out), 2), (p(b), p(ip), 1, None, 2), (p(b), p(ip), 1, p(out), -1),
                 (p(b), p(bad), 2, p(out), 2), (p(b), p(np.array([1, 64], np.int32)), 1, p(out), 2)):
        assert L.tkv_plan_row_blocks(*args) == tkv.TKV_ERR_INVALID_ARG


# ------------------------------------------------------------------ what the bindings take (CPU tensors; prepare=True launches nothing)
def rows(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype)


def bound_prefill(**kw):
    a = dict(q=rows(3, 4, 128), K=rows(3, 2, 128), V=rows(3, 2, 128), kp=rows(5, 2, 128, dtype=torch.float16), vp=rows(5, 2, 128, dtype=torch.float16), out=rows(3, 4, 128))
    a.update(kw)
    pf = tkv.tkv_prefill.make(plan([3], [5], 4, 2), "cpu")
    return tkv.tkv_prefill_attention(tkv.tkv_desc.make(2, 0, 0), a["q"], a["K"], a["V"], a["kp"], a["vp"], pf, 0.1, a["out"], rows(16, dtype=torch.uint8), stream=0, prepare=True)


def test_bindings_take_what_they_say():
    bound_prefill()
    bound_prefill(K=rows(3, 2, 128, dtype=torch.float16), V=rows(3, 2, 128, dtype=torch.float16), out=rows(3, 4, 128, dtype=torch.float16))
    packed = rows(3, 8, 128)
    bound_prefill(q=packed[:, :4], K=packed[:, 4:6], V=packed[:, 6:])
    bound_prefill(kp=None, vp=None)


@pytest.mark.parametrize("kw", [dict(q=rows(3, 4, 128, dtype=torch.float32)), dict(q=rows(3, 4, 64)), dict(q=rows(3, 512)), dict(K=rows(3, 2, 128, dtype=torch.float16)),
                                dict(K=rows(2, 2, 128)), dict(V=rows(3, 3, 128)), dict(V=rows(3, 2, 128, dtype=torch.int16)), dict(kp=rows(5, 2, 128)), dict(kp=None),
                                dict(vp=rows(4, 2, 128, dtype=torch.float16)), dict(kp=rows(5, 4, 128, dtype=torch.float16)[:, ::2]), dict(out=rows(3, 4, 128, dtype=torch.float32)),
                                dict(out=rows(4, 4, 128)), dict(out=rows(3, 8, 128)[:, :4]), dict(q=rows(3, 128, 4).transpose(1, 2)), dict(K=rows(3, 4, 128)[:, ::2])])
def test_the_binding_of_prompt_attention_refuses(kw):
    with pytest.raises(AssertionError):
        bound_prefill(**kw)


@pytest.mark.parametrize("kw", [dict(K=rows(40, 2, 128, dtype=torch.float16)), dict(V=rows(41, 2, 128)), dict(bits=rows(40, dtype=torch.int32)), dict(bits=rows(39, dtype=torch.uint8)),
                                dict(blocks=rows(32, dtype=torch.float32)), dict(blocks=rows(33, dtype=torch.int32)), dict(ko=rows(40, 2, 128)), dict(vo=rows(40, 3, 128, dtype=torch.float16))])
def test_the_binding_of_rows_refuses(kw):
    half = lambda: rows(40, 2, 128, dtype=torch.float16)  # noqa: E731
    a = dict(K=rows(40, 2, 128), V=rows(40, 2, 128), bits=rows(40, dtype=torch.uint8), blocks=None, ko=half(), vo=half())
    call = lambda: tkv.tkv_quantize_rows(tkv.tkv_desc.make(2, 0, 0, int2_key_axis=1), *a.values(), stream=0, prepare=True)  # noqa: E731
    call()
    a.update(kw)
    with pytest.raises(AssertionError):
        call()


@pytest.mark.parametrize("kw", [dict(y=rows(9, 2, 128, dtype=torch.float16)), dict(y=rows(8, 2, 128)), dict(x=rows(9, 2, 64), y=rows(9, 2, 64)), dict(ip=rows(3, dtype=torch.int64)),
                                dict(out=rows(2, 2, dtype=torch.float32)), dict(out=rows(3, 2, dtype=torch.float64)), dict(x=rows(9, 2, 128, dtype=torch.int16), y=rows(9, 2, 128, dtype=torch.int16))])
def test_the_binding_of_distortion_refuses(kw):
    a = dict(x=rows(9, 2, 128), y=rows(9, 2, 128), ip=rows(3, dtype=torch.int32), out=rows(2, 2, dtype=torch.float64), ws=rows(4096, dtype=torch.uint8))
    call = lambda: tkv.tkv_head_distortion(*a.values(), stream=0, prepare=True)  # noqa: E731
    call()
    a.update(kw)
    with pytest.raises(AssertionError):
        call()
