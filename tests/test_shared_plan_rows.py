"""The rows of a plan's items travel as a field of the plan and an argument of their own."""
import pytest
import torch

from paper_2605_17170_amd import tkv


def parts(plan):
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    return (i32(2), i32(40), i32(1), i32(1), i32(2), i32(len(plan.member_slots)), torch.from_numpy(plan.member_slots), torch.from_numpy(plan.prefix_items))


@pytest.mark.parametrize("seqs,tokens", [(1, 64), (4, 20000), (40, 40000)])
def test_tile_rows_of_plan_and_prefix(seqs, tokens):
    desc = tkv.tkv_desc.make(4, 1000, 1000)
    plan = tkv.tkv_plan_decode_shared(desc, seqs, 32, [tokens], [tokens], [0, seqs], list(range(seqs)), 256, [], [0] * (seqs + 1))
    assert plan.tile_rows in (16, 64, 128) and plan.tile_rows == plan.max_members.tile_rows
    assert tkv.tkv_prefix.make(*parts(plan), tile_rows=plan.tile_rows).tile_rows == plan.tile_rows
    assert tkv.tkv_prefix.make(*parts(plan), plan.max_members).tile_rows == plan.tile_rows
    assert tkv.tkv_prefix.make(*parts(plan), int(plan.max_members), tile_rows=plan.tile_rows).tile_rows == plan.tile_rows
    for given in (dict(), dict(max_members=16), dict(max_members=int(plan.max_members)), dict(tile_rows=32), dict(tile_rows=0)):
        with pytest.raises(ValueError):
            tkv.tkv_prefix.make(*parts(plan), **given)
