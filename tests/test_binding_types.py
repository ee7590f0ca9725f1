"""The bindings of norm and rotation, page tables and shared prefixes refuse tensors whose bits mean something else: fp16 rows for
bf16, 32-bit floats for whole numbers.  CPU tensors; nothing is launched (prepare=True)."""
import pytest
import torch

from paper_2605_17170_amd import tkv

DESC = tkv.tkv_desc.make(1, 4, 4)


def i32(*shape, dtype=torch.int32):
    return torch.zeros(shape, dtype=dtype)


def rows(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype)


def norm_rope(**kw):
    a = dict(q=rows(3, 2, 128), k=rows(3, 1, 128), v=rows(3, 1, 128), pos=i32(1, 3), wq=rows(128), wk=rows(128), qo=rows(3, 2, 128), ko=rows(3, 1, 128),
             vo=rows(3, 1, 128))
    a.update(kw)
    rope = tkv.tkv_rope_make(128, device="cpu")
    return tkv.tkv_norm_rope(rope, a["q"], a["k"], a["v"], a["pos"], a["wq"], a["wk"], 1e-6, a["qo"], a["ko"], a["vo"], stream=0, prepare=True)


def table(**kw):
    a = dict(rows=i32(2, 4), n2=i32(2), n4=i32(2), free=i32(8), n_free=i32(2), keep=i32(2), lens=i32(2), tags=torch.zeros(5, dtype=torch.uint8), indptr=i32(3),
             pos=i32(5), slots=i32(5), pages=i32(5), src=i32(5, 64), n_work=i32(1))
    a.update(kw)
    t = tkv.tkv_table.make(a["rows"], a["n2"], a["n4"], a["free"], a["n_free"])
    return tkv.tkv_table_append(DESC, t, a["keep"], a["keep"], a["lens"], a["tags"], a["indptr"], a["pos"], a["slots"], a["pages"], a["src"], a["n_work"],
                                torch.zeros(4096, dtype=torch.uint8), stream=0, prepare=True)


def shared(**kw):
    plan = tkv.tkv_plan_decode_shared(DESC, 2, 2, [100], [70], [0, 2], [0, 1], 4, [[0, 0, 1, 0]], [0, 1, 1])
    a = dict(q=rows(2, 2, 128), out=rows(2, 2, 128), indptr=i32(3), ids=i32(8), n2=i32(2), n4=i32(2), items=torch.from_numpy(plan.items),
             slots=torch.from_numpy(plan.seq_item_indptr), p_ids=i32(8), p_n2=i32(1), members=i32(2))
    a.update(kw)
    prefix = tkv.tkv_prefix.make(i32(2), a["p_ids"], a["p_n2"], i32(1), i32(2), a["members"], torch.from_numpy(plan.member_slots),
                                 torch.from_numpy(plan.prefix_items), plan.max_members)
    pool, bit_map = torch.zeros(tkv.tkv_pool_bytes(DESC), dtype=torch.uint8), torch.zeros(8, dtype=torch.uint8)
    return tkv.tkv_decode_attention_shared(DESC, pool, bit_map, a["q"], a["indptr"], a["ids"], a["n2"], a["n4"], a["items"], prefix, a["slots"], plan.n_slots, 0.1,
                                           a["out"], torch.zeros(1 << 16, dtype=torch.uint8), stream=0, prepare=True)


HALF, FLOAT = torch.float16, torch.float32


def test_the_right_types_and_raw_patterns_pass():
    for call in (norm_rope, table, shared):
        assert call() is not None
    assert norm_rope(q=rows(3, 2, 128, dtype=torch.int16), wk=rows(128, dtype=torch.int16)) is not None


@pytest.mark.parametrize("call,kw", [
    (norm_rope, dict(q=rows(3, 2, 128, dtype=HALF))), (norm_rope, dict(v=rows(3, 1, 128, dtype=HALF))), (norm_rope, dict(ko=rows(3, 1, 128, dtype=HALF))),
    (norm_rope, dict(wq=rows(128, dtype=HALF))), (norm_rope, dict(pos=i32(1, 3, dtype=FLOAT))), (norm_rope, dict(pos=i32(1, 3, dtype=torch.int64))),
    (table, dict(rows=i32(2, 4, dtype=FLOAT))), (table, dict(keep=i32(2, dtype=FLOAT))), (table, dict(lens=i32(2, dtype=FLOAT))),
    (table, dict(src=i32(5, 64, dtype=FLOAT))), (table, dict(n_work=i32(1, dtype=FLOAT))),
    (shared, dict(q=rows(2, 2, 128, dtype=HALF))), (shared, dict(out=rows(2, 2, 128, dtype=HALF))), (shared, dict(ids=i32(8, dtype=FLOAT))),
    (shared, dict(ids=i32(8, dtype=torch.int64))), (shared, dict(n2=i32(2, dtype=FLOAT))), (shared, dict(p_n2=i32(1, dtype=FLOAT))),
])
def test_other_types_are_refused(call, kw):
    with pytest.raises(AssertionError):
        call(**kw)
