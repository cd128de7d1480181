"""Arrays of 32-bit numbers that do not start on a 4-byte boundary are refused before anything is launched."""
import ctypes as C

import pytest
import torch

from paper_2605_07230_b200 import binding as cb
from tests import gpu_util as G
from tests.test_gpu_paged import make_ctx

pytestmark = pytest.mark.gpu


def each_shifted(args, arrays):
    """args with one of the arrays moved by 1 to 3 bytes, the others where they were."""
    for i in arrays:
        for d in (1, 2, 3):
            yield (i, d), [a + d if k == i else a for k, a in enumerate(args)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_misaligned_arrays_are_refused(dtype):
    L = cb.lib()
    ctx = make_ctx(dtype, 2, 2, 64)
    buf = torch.zeros(1 << 16, dtype=torch.int32, device=G.DEV)
    at = [buf.data_ptr() + 4096 * i for i in range(16)]
    tables = [1, 1, 8, 4, *at[:3], 2, *at[3:5], *at[5:8], *at[8:10], None]
    slots = [4, 5, 6, 8, 9, 10, 11, 12, 13, 14]
    assert [tables[i] for i in slots] == at[:10]
    for what, args in each_shifted(tables, slots):
        assert L.cascade_paged_tables(ctx.handle, *args) == cb.ERR_INVALID_ARG, what

    def cache(d=0):
        return C.byref(cb.PagedCacheStruct(at[0], at[4], 1024, 1, 8, at[8] + d, 2))

    append = [1, None, 0, at[9], 128, at[10], 128, at[11], at[12], 0.0, None, 0, None]
    for what, args in each_shifted(append, [7, 8]):
        assert L.cascade_paged_append(ctx.handle, cache(), *args) == cb.ERR_INVALID_ARG, what
    attn = [1, 1, at[9], 128, at[10], at[11], 1, 8, 0, 0, 1.0, at[12], at[13], None]
    for what, args in each_shifted(attn, [4, 5, 12]):
        assert L.cascade_paged_attn(ctx.handle, cache(), *args) == cb.ERR_INVALID_ARG, what
    for d in (1, 2, 3):
        assert L.cascade_paged_attn(ctx.handle, cache(d), *attn) == cb.ERR_INVALID_ARG, d
    sample = [at[0], cb.F32, 64, 1, *at[1:9], None]
    for what, args in each_shifted(sample, range(4, 12)):
        assert L.cascade_sample(ctx.handle, *args) == cb.ERR_INVALID_ARG, what
    torch.cuda.synchronize()
    assert int(buf.abs().sum()) == 0
    assert L.cascade_paged_append(ctx.handle, cache(), *append) == cb.OK
    assert L.cascade_paged_attn(ctx.handle, cache(), *attn) == cb.OK
    assert L.cascade_sample(ctx.handle, *sample) == cb.OK
    torch.cuda.synchronize()
    ctx.check()
    ctx.close()
