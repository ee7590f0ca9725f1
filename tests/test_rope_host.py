"""Rotation table and the refusals of tkv_norm_rope that need no GPU: nothing here launches anything."""
import ctypes as C
import math
from fractions import Fraction

import numpy as np
import pytest

from paper_2605_17170_amd import tkv


def turns(word):
    return (int(word) & ~3) / 2.0 ** 64


@pytest.mark.parametrize("rotary,theta", [(128, 1e4), (128, 5e6), (64, 1e6), (16, 2.0)])
def test_words_are_turns_per_position(rotary, theta):
    table = tkv.tkv_rope_table(rotary, theta)
    want = np.array([theta ** (-2.0 * i / rotary) / (2 * math.pi) for i in range(rotary // 2)])
    # 2^-63 turns by the axis bits, a few units in the last place of the 64-bit reference
    assert np.all(np.abs(np.array([turns(w) for w in table]) - want) <= 2.0 ** -62 + 1e-15 * want)
    assert all(int(w) & 3 == 0 for w in table)


@pytest.mark.parametrize("sections,interleaved,want", [
    ([2, 3, 3], False, [0, 0, 1, 1, 1, 2, 2, 2]),
    ([4, 2, 2], True, [0, 1, 2, 0, 1, 2, 0, 0]),
    ([0, 0, 8, 0], False, [2] * 8),
    ([3, 3, 2], True, [0, 1, 2, 0, 1, 2, 0, 1]),
    ([4, 4], True, [0, 1] * 4),
    ([8], True, [0] * 8),
])
def test_axis_of_each_pair(sections, interleaved, want):
    table = tkv.tkv_rope_table(16, 100.0, sections, interleaved)
    assert [int(w) & 3 for w in table] == want


def test_frequencies_given_by_the_caller_negative_and_above_one_turn():
    f = [0.0, 0.5, -0.5, 7.0, 2 * math.pi * 0.75, 1e-9, -1e-9, 6.0]
    table = tkv.tkv_rope_table(16, inv_freq=f)
    for w, x in zip(table, f):
        want = Fraction(x) / Fraction("6.283185307179586476925286766559005768")
        off = abs(Fraction(int(w) & ~3, 2 ** 64) - want)
        off -= math.floor(off)
        assert min(off, 1 - off) <= Fraction(1, 2 ** 61)


@pytest.mark.parametrize("kw,status", [
    (dict(rotary_dim=8), tkv.TKV_ERR_BAD_SHAPE), (dict(rotary_dim=130), tkv.TKV_ERR_BAD_SHAPE), (dict(rotary_dim=-16), tkv.TKV_ERR_BAD_SHAPE),
    (dict(rotary_dim=16, sections=[1, 2]), tkv.TKV_ERR_BAD_SHAPE), (dict(rotary_dim=16, sections=[9, -1]), tkv.TKV_ERR_BAD_SHAPE),
    (dict(rotary_dim=16, sections=[2, 2, 2, 1, 1]), tkv.TKV_ERR_BAD_SHAPE),
    (dict(rotary_dim=16, sections=[2, 3, 3], interleaved=True), tkv.TKV_ERR_BAD_SHAPE),   # the third axis has two turns
    (dict(rotary_dim=16, theta=0.0), tkv.TKV_ERR_INVALID_ARG), (dict(rotary_dim=16, theta=float("nan")), tkv.TKV_ERR_INVALID_ARG),
    (dict(rotary_dim=16, inv_freq=[1, 2, 3, 4, 5, 6, 7, float("inf")]), tkv.TKV_ERR_INVALID_ARG),
])
def test_table_refusals(kw, status):
    with pytest.raises(tkv.TkvError) as e:
        tkv.tkv_rope_table(**kw)
    assert e.value.status == status


def call(**kw):
    """tkv_norm_rope with host addresses that are never touched."""
    a = dict(rope=tkv.tkv_rope(128, 1, 0, 1.0, 256), q=4096, qs=512, k=8192, ks=128, v=12288, vs=128, n=3, hq=4, hk=1, pos=64, wq=256, wk=512,
             eps=1e-6, qo=16384, ko=32768, vo=65536)
    a.update(kw)
    rope = C.byref(a["rope"]) if a["rope"] is not None else None
    return tkv.lib().tkv_norm_rope(rope, a["q"], a["qs"], a["k"], a["ks"], a["v"], a["vs"], a["n"], a["hq"], a["hk"], a["pos"], a["wq"], a["wk"],
                                   a["eps"], a["qo"], a["ko"], a["vo"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(rope=None), tkv.TKV_ERR_INVALID_ARG),
    (dict(rope=tkv.tkv_rope(24, 1, 0, 1.0, 256)), tkv.TKV_ERR_BAD_SHAPE),
    (dict(rope=tkv.tkv_rope(144, 1, 0, 1.0, 256)), tkv.TKV_ERR_BAD_SHAPE),
    (dict(rope=tkv.tkv_rope(128, 5, 0, 1.0, 256)), tkv.TKV_ERR_BAD_SHAPE),
    (dict(rope=tkv.tkv_rope(128, 1, 2, 1.0, 256)), tkv.TKV_ERR_INVALID_ARG),
    (dict(rope=tkv.tkv_rope(128, 1, 0, float("nan"), 256)), tkv.TKV_ERR_INVALID_ARG),
    (dict(rope=tkv.tkv_rope(128, 1, 0, 1.0, None)), tkv.TKV_ERR_INVALID_ARG),
    (dict(rope=tkv.tkv_rope(128, 1, 0, 1.0, 260)), tkv.TKV_ERR_INVALID_ARG),
    (dict(pos=None), tkv.TKV_ERR_INVALID_ARG),
    (dict(n=-1), tkv.TKV_ERR_INVALID_ARG), (dict(hq=-1), tkv.TKV_ERR_INVALID_ARG), (dict(hk=-1), tkv.TKV_ERR_INVALID_ARG),
    (dict(eps=-1e-6), tkv.TKV_ERR_INVALID_ARG), (dict(eps=float("nan")), tkv.TKV_ERR_INVALID_ARG),
    (dict(q=None), tkv.TKV_ERR_INVALID_ARG), (dict(qo=None), tkv.TKV_ERR_INVALID_ARG), (dict(vo=None), tkv.TKV_ERR_INVALID_ARG),
    (dict(q=4098), tkv.TKV_ERR_INVALID_ARG), (dict(ko=32776), tkv.TKV_ERR_INVALID_ARG), (dict(wq=264), tkv.TKV_ERR_INVALID_ARG),
    (dict(qs=516), tkv.TKV_ERR_INVALID_ARG), (dict(qs=504), tkv.TKV_ERR_INVALID_ARG), (dict(ks=0), tkv.TKV_ERR_INVALID_ARG),
    (dict(q=4096, qo=4096, qs=1024), tkv.TKV_ERR_INVALID_ARG),                 # in place only where the input is contiguous
    (dict(n=1 << 20, hq=4096, qs=4096 * 128), tkv.TKV_ERR_INVALID_ARG),
    (dict(n=0), tkv.TKV_OK), (dict(hq=0, hk=0, v=None), tkv.TKV_OK),
])
def test_calls_that_launch_nothing(kw, status):
    assert call(**kw) == status
