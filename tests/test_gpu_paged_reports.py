"""Slots and pages outside their range are reported by the call that meets them."""
import pytest
import torch

from paper_2605_07230_b200 import binding as cb
from oracle import paged_oracle as PO
from tests import gpu_util as G
from tests.test_gpu_paged import i32, make_ctx, run_tables

pytestmark = pytest.mark.gpu


def reports_bad_page(ctx):
    with pytest.raises(cb.CascadeError) as e:
        ctx.check()
    return e.value.status == cb.ERR_BAD_PAGE


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("slot", [-2, -17, -2 ** 31, 16])
def test_append_reports_every_slot_that_is_neither_in_the_pool_nor_minus_one(dtype, slot):
    ctx = make_ctx(dtype, 4, 2, 64)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    pool = torch.zeros(2, 2, 8, 2, 64, dtype=dt, device=G.DEV)
    cache = cb.PagedCache(pool[0], pool[1], i32([[0]]))
    k = torch.ones(3, 2, 64, dtype=dt, device=G.DEV)
    cb.cascade_paged_append(ctx, cache, k, k, i32([3, -1, 5]), i32([0, 0, 1]))
    ctx.check()
    assert float(pool.float().sum()) == 4 * 128
    cb.cascade_paged_append(ctx, cache, k, k, i32([3, slot, 5]), i32([0, 0, 1]))
    assert reports_bad_page(ctx)
    assert float(pool.float().sum()) == 4 * 128
    ctx.close()


@pytest.mark.parametrize("page", [-1, 6, 10 ** 9])
def test_tables_report_a_bad_page_that_is_given_back(page):
    ctx = make_ctx()
    args = ([-1, 0], [17, 8], [[4, page, 1], [2, -1, -1]], [3, -5, -5, -5, -5, -5], 1)
    got = run_tables(ctx, *args, 8, 2)
    assert reports_bad_page(ctx)
    ref = PO.tables(*args, 8, 2)                     # the stack's count and order hold; the entry is the caller's own
    assert got["free"].tolist() == ref["free"].tolist() and int(got["count"]) == ref["count"] == 4
    got = run_tables(ctx, [-1, 0], [17, 8], [[4, 0, 1], [2, -1, -1]], [3, -5, -5, -5, -5, -5], 1, 8, 2)
    ctx.check()
    ctx.close()
