"""What the binding hands to the library for block tables that are parts of wider ones (CPU)."""
import ctypes as C

import pytest
import torch

from paper_2605_07230_b200 import binding as cb


def table_fields(table):
    pool = torch.zeros(3, 8, 2, 64, dtype=torch.bfloat16)
    s = cb.PagedCache(pool, pool.clone(), table).struct
    return s.table_stride, s.table_width


@pytest.mark.parametrize("rows,columns,first,width", [(4, 20, 0, 6), (4, 20, 3, 17), (2, 5, 0, 5), (1, 9, 2, 4), (3, 7, 6, 1)])
def test_a_slice_of_a_table_keeps_its_own_width(rows, columns, first, width):
    table = torch.zeros(rows, columns, dtype=torch.int32)[:, first: first + width]
    stride, got = table_fields(table)
    assert got == width and stride == (columns if rows > 1 else width)
    # the last entry that a request may name lies in the table's own memory
    last = (rows - 1) * stride + got - 1
    assert first + last < rows * columns


def test_a_table_without_columns_has_no_entries():
    for table in (torch.zeros(3, 0, dtype=torch.int32), torch.zeros(3, 5, dtype=torch.int32)[:, :0]):
        assert table_fields(table) == (0, 0)                     # refused: a table_stride below 1


def test_struct_layout_is_the_header_s():
    assert C.sizeof(cb.PagedCacheStruct) == 48 and cb.PagedCacheStruct.table_width.offset == 44
