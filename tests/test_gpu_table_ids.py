"""Page ids that cannot be: tkv_table_append hands on what rows and free lists hold, and append leaves such pages out."""
import numpy as np
import pytest
import torch

from paper_2605_17170_amd import tkv

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("n_seqs", [3, 1030])     # one launch, and four
def test_ids_are_handed_on_and_append_leaves_them_out(n_seqs):
    p2, p4 = 8, n_seqs + 8
    desc = tkv.tkv_desc.make(1, p2, p4)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device=DEV)  # noqa: E731
    table = tkv.tkv_table.make(i32(n_seqs, 4), i32(n_seqs), i32(n_seqs), i32(p2 + p4), i32(2))
    tkv.tkv_table_reset(desc, table)
    rows, _, n4, free, n_free = table.tensors
    top = p2 + int(n_free[1]) - 1
    good = int(free[top - 2])
    free[top], free[top - 1] = -1, 3                # none, and one of the other width, to sequences 0 and 1
    lens, tags = torch.ones(n_seqs, dtype=torch.int32, device=DEV), torch.full((n_seqs,), 4, dtype=torch.uint8, device=DEV)
    work = tkv.tkv_table_max_work(n_seqs, n_seqs)
    slots, pages, src, status = i32(n_seqs), i32(work), i32(work, 64), i32(1)
    ws = torch.empty(tkv.tkv_table_workspace_bytes(n_seqs, n_seqs), dtype=torch.uint8, device=DEV)
    tkv.tkv_table_append(desc, table, None, None, lens, tags, None, None, slots, pages, src, i32(1), ws, status)
    torch.cuda.synchronize()
    assert int(status.item()) == 0 and pages[:3].tolist() == [-1, 3, good] and slots[:3].tolist() == [-64, 192, 64 * good]
    assert rows[:3, 0].tolist() == [-1, 3, good] and n4.tolist() == [1] * n_seqs
    pool, bit_map = torch.full((tkv.tkv_pool_bytes(desc),), 0x5A, dtype=torch.uint8, device=DEV), torch.zeros(p2 + p4, dtype=torch.uint8, device=DEV)
    k = torch.ones((n_seqs, 1, 128), dtype=torch.bfloat16, device=DEV)
    tkv.tkv_quantize_append(desc, pool, bit_map, k, k, tags, pages, src, status)
    torch.cuda.synchronize()
    assert int(status.item()) == tkv.TKV_STATUS_PAGE_RANGE | tkv.TKV_STATUS_TAG_MISMATCH
    assert bit_map[:p2].tolist() == [0] * p2 and bool((pool[:p2 * tkv.tkv_page_bytes(desc, 2)] == 0x5A).all())
    assert int(bit_map[good]) == 4 and int((bit_map == 4).sum()) == n_seqs - 2
    # given back, they are what the free list holds again
    keep = i32(n_seqs)
    tkv.tkv_table_append(desc, table, keep, keep, None, None, None, None, None, None, None, i32(1), ws, status.zero_())
    torch.cuda.synchronize()
    assert int(status.item()) == 0 and free[top - 2:top + 1].tolist() == [good, 3, -1] and int(n_free[1]) == p4
    assert np.all(rows.cpu().numpy() == -1)
