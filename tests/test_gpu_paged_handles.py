"""Views that a handle of the paged operators must not take: the library would read other memory than the tensor's."""
import pytest
import torch

import paper_2512_14481_b200 as P

pytestmark = pytest.mark.gpu


def i32(a):
    return torch.tensor(a, dtype=torch.int32, device="cuda")


def test_page_tables_whose_rows_overlap_are_refused():
    lens, starts = i32([20, 20, 20]), i32([0, 1, 2, 3])
    shared = i32([[0, 1]]).expand(3, -1)                       # strides (0, 1)
    sliding = torch.as_strided(i32([0, 1, 2, 3]), (3, 2), (1, 1))
    narrow = i32([[0]]).expand(3, 1)                           # one page each, all the same entry
    for table in (shared, sliding, narrow):
        with pytest.raises(ValueError):
            P.PagedBatch(table, lens, starts, 3)
    # a copy is fine, and so are rows further apart than they are wide, and one row of any stride
    assert P.PagedBatch(shared.contiguous(), lens, starts, 3).struct.page_table_stride == 2
    wide = torch.zeros((3, 5), dtype=torch.int32, device="cuda")
    assert P.PagedBatch(wide[:, :2], lens, starts, 3).struct.page_table_stride == 5
    one = torch.as_strided(i32([0, 1]), (1, 2), (1, 1))
    assert P.PagedBatch(one, i32([20]), i32([0, 1]), 1).struct.page_table_stride == 2
