"""Slots and pages outside their range are reported by the call that meets them."""
import pytest
import torch

from paper_2605_07230_b200 import binding as cb
from tests import gpu_util as G
from tests.test_gpu_paged import i32, make_ctx

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
