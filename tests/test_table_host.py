"""The model of tkv_table_append against the host planner, and the refusals of the entry points that need no GPU."""
import ctypes as C

import numpy as np
import pytest

from paper_2605_17170_amd import tkv
from table_model import Table


@pytest.mark.parametrize("key_axis", [0, 1])
def test_the_model_is_the_host_planner_sequence_by_sequence(key_axis):
    rng = np.random.default_rng(7 + key_axis)
    n, p2, p4 = 5, 90, 90
    desc = tkv.tkv_desc.make(2, p2, p4, int2_key_axis=key_axis)
    alloc, seqs = tkv.tkv_alloc_create(desc), [tkv.tkv_seq_create() for _ in range(n)]
    model = Table(n, 200, p2, p4)
    for step in range(6):
        chunks = [rng.choice([2, 4], rng.integers(0, 300)).astype(np.uint8) for _ in range(n)]
        if key_axis:
            chunks = [tkv.tkv_route_residual(c) for c in chunks]
        tags = np.concatenate(chunks)
        got = model.append(None, [c.size for c in chunks], tags, key_axis == 1)
        base, at = 0, 0
        for b in range(n):
            slots, pages, src = tkv.tkv_plan_append(alloc, seqs[b], chunks[b], base)
            assert np.array_equal(got["slots"][base:base + slots.size], slots)
            assert np.array_equal(got["work_pages"][at:at + pages.size], pages) and np.array_equal(got["work_src"][at:at + pages.size], src)
            base, at = base + slots.size, at + pages.size
            ids = tkv.tkv_seq_page_ids(seqs[b])
            assert np.array_equal(model.rows()[b, :ids.size], ids) and np.all(model.rows()[b, ids.size:] == -1)
        assert at == got["work_pages"].size <= tkv.tkv_table_max_work(n, tags.size)
    for s in seqs:
        tkv.tkv_seq_destroy(s)
    tkv.tkv_alloc_destroy(alloc)


def test_what_is_appended_again_after_a_cut_gets_the_same_pages():
    rng = np.random.default_rng(3)
    model = Table(4, 100, 60, 60)
    model.append(None, [100, 0, 257, 64], rng.choice([2, 4], 421))
    keep = [list(c) for c in model.count]
    tags = rng.choice([2, 4], 600)
    first = model.append(None, [150, 150, 150, 150], tags)
    free = [list(f) for f in model.free]
    again = model.append(keep, [150, 150, 150, 150], tags)
    assert all(np.array_equal(first[k], again[k]) for k in first) and free == model.free


def test_bounds_of_the_work_list():
    assert tkv.tkv_table_max_work(32, 32) == 32 and tkv.tkv_table_max_work(0, 0) == 0
    assert tkv.tkv_table_max_work(1, 65536) == 1028 and tkv.tkv_table_max_work(8, 3) == 3
    for a, b in ((-1, 4), (4, -1), (4, (1 << 28) + 1)):
        with pytest.raises(tkv.TkvError):
            tkv.tkv_table_max_work(a, b)
        assert tkv.tkv_table_workspace_bytes(a, b) == 0


DESC = tkv.tkv_desc.make(2, 10, 10)


def call(**kw):
    """tkv_table_append with addresses that are never touched."""
    a = dict(desc=DESC, table=tkv.tkv_table(4, 16, 4096, 8192, 8256, 12288, 16384), keep2=64, keep4=64, n_new=64, tags=64, n_tokens=4, indptr=64,
             positions=64, slots=64, pages=64, src=64, max_work=4, n_work=64, ws=256, ws_bytes=1 << 20, status=64)
    a.update(kw)
    by = lambda x: C.byref(x) if x is not None else None  # noqa: E731
    return tkv.lib().tkv_table_append(by(a["desc"]), by(a["table"]), a["keep2"], a["keep4"], a["n_new"], a["tags"], a["n_tokens"], a["indptr"],
                                      a["positions"], a["slots"], a["pages"], a["src"], a["max_work"], a["n_work"], a["ws"], a["ws_bytes"],
                                      a["status"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(desc=None), tkv.TKV_ERR_INVALID_ARG), (dict(desc=tkv.tkv_desc.make(0, 1, 1)), tkv.TKV_ERR_BAD_SHAPE),
    (dict(table=None), tkv.TKV_ERR_INVALID_ARG),
    (dict(table=tkv.tkv_table(-1, 16, 64, 64, 64, 64, 64)), tkv.TKV_ERR_INVALID_ARG),
    (dict(table=tkv.tkv_table(4, -1, 64, 64, 64, 64, 64)), tkv.TKV_ERR_INVALID_ARG),
    (dict(table=tkv.tkv_table(4, (1 << 24) + 1, 64, 64, 64, 64, 64)), tkv.TKV_ERR_INVALID_ARG),
    (dict(table=tkv.tkv_table(1 << 20, 1 << 12, 64, 64, 64, 64, 64)), tkv.TKV_ERR_INVALID_ARG),
    (dict(table=tkv.tkv_table(4, 16, None, 64, 64, 64, 64)), tkv.TKV_ERR_INVALID_ARG),
    (dict(table=tkv.tkv_table(4, 16, 64, None, 64, 64, 64)), tkv.TKV_ERR_INVALID_ARG),
    (dict(table=tkv.tkv_table(4, 16, 64, 64, 64, None, 64)), tkv.TKV_ERR_INVALID_ARG),
    (dict(table=tkv.tkv_table(4, 16, 64, 64, 64, 64, None)), tkv.TKV_ERR_INVALID_ARG),
    (dict(table=tkv.tkv_table(4, 16, 66, 64, 64, 64, 64)), tkv.TKV_ERR_INVALID_ARG),
    (dict(n_tokens=-1), tkv.TKV_ERR_INVALID_ARG), (dict(n_tokens=(1 << 28) + 1), tkv.TKV_ERR_INVALID_ARG), (dict(max_work=-1), tkv.TKV_ERR_INVALID_ARG),
    (dict(tags=None), tkv.TKV_ERR_INVALID_ARG), (dict(pages=None), tkv.TKV_ERR_INVALID_ARG), (dict(src=None), tkv.TKV_ERR_INVALID_ARG),
    (dict(n_work=None), tkv.TKV_ERR_INVALID_ARG), (dict(ws=None), tkv.TKV_ERR_INVALID_ARG), (dict(ws=264), tkv.TKV_ERR_INVALID_ARG),
    (dict(slots=65), tkv.TKV_ERR_INVALID_ARG), (dict(keep4=66), tkv.TKV_ERR_INVALID_ARG), (dict(status=67), tkv.TKV_ERR_INVALID_ARG),
    (dict(ws_bytes=16), tkv.TKV_ERR_WORKSPACE_TOO_SMALL),
])
def test_calls_that_launch_nothing(kw, status):
    assert call(**kw) == status


def test_reset_refuses_what_append_refuses():
    t = tkv.tkv_table(4, 16, 64, 64, 64, 64, None)
    assert tkv.lib().tkv_table_reset(C.byref(DESC), C.byref(t), None) == tkv.TKV_ERR_INVALID_ARG
    assert tkv.lib().tkv_table_reset(None, C.byref(t), None) == tkv.TKV_ERR_INVALID_ARG
