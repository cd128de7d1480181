"""Block tables that are columns of wider ones: results as with a table of their own, lengths past their width left out."""
import ctypes as C

import pytest
import torch

from paper_2605_07230_b200 import binding as cb
from tests import gpu_util as G
from tests.test_gpu_paged import Case, DT, make_ctx

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("q", [1, 40])
def test_columns_of_a_wider_table(dtype, q):
    ctx = make_ctx(dtype, 4, 2, 64)
    c = Case(dtype, 4, 2, 64, 16, [q] * 4, [q + 50, q + 9, q + 44, q + 60], extra_width=0)
    n, width = c.table.shape
    wide = torch.zeros(n, 3 * width, dtype=torch.int32, device=G.DEV)          # page 0 on both sides
    wide[:, width: 2 * width] = c.cache.block_table
    c.cache = cb.PagedCache(c.kp, c.vp, wide[:, width: 2 * width])
    c.run(ctx)
    ctx.check()
    c.check()
    c.out.fill_(3.0)
    c.lse.fill_(3.0)
    for r in (1, 3):                                             # inside the wider table, past the slice
        c.kv[r] = 16 * width + 1
    c.run(ctx, max_kv=16 * width * 2)
    with pytest.raises(cb.CascadeError) as e:
        ctx.check()
    assert e.value.status == cb.ERR_BAD_PAGE
    c.check(requests=[0, 2])
    for r in (1, 3):
        assert (c.out[r * q: (r + 1) * q] == 3).all() and (c.lse[r * q: (r + 1) * q] == 3).all()
    ctx.close()


def test_widths_that_are_refused():
    L = cb.lib()
    ctx = make_ctx("bf16", 2, 2, 64)
    buf = torch.zeros(8192, dtype=torch.bfloat16, device=G.DEV)
    idx = torch.zeros(64, dtype=torch.int32, device=G.DEV)
    p, i = buf.data_ptr(), idx.data_ptr()

    def call(stride, width):
        cache = cb.PagedCacheStruct(p + 4096, p + 8192, 8 * 128, 1, 8, i, stride, width)
        return L.cascade_paged_attn(ctx.handle, C.byref(cache), 1, 1, p, 128, i, i, 1, 8, 0, 0, 1.0, p + 1024, None, None)

    for stride, width in ((4, -1), (4, 5), (0, 0), (0, 1), (-1, 0)):
        assert call(stride, width) == cb.ERR_INVALID_ARG, (stride, width)
    for stride, width in ((4, 0), (4, 4), (4, 1)):
        assert call(stride, width) == cb.OK, (stride, width)
    torch.cuda.synchronize()
    ctx.check()
    ctx.close()
