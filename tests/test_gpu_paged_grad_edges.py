"""GPU: rows that see no key beside keys that hold no numbers, in the paged attention's gradient."""
import numpy as np
import pytest
import torch

from paper_2605_07230_b200 import binding as cb
from tests import gpu_util as G
from tests.test_gpu_paged_grad import Call

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,Hkv", [(2, 2), (5, 1)])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("where", ["key", "value"])
def test_rows_without_keys_beside_a_key_that_is_no_number(where, value, Hq, Hkv, D, dtype):
    """Fewer keys than new tokens: the first rows see nothing, whatever the keys of their block hold."""
    q_len, kv_len = [7, 140, 30], [2, 100, 30]
    c = Call(q_len, kv_len, Hq, Hkv, D, dtype, seed=31, pad=1)
    pool = c.k_pages if where == "key" else c.v_pages
    for r, j in ((0, 1), (1, 60)):                                   # seen by the last row, and by the last forty
        pool[int(c.table_host[r, j // 16]), j % 16, :, 5] = value
    c.run()
    for r, (n, kv, j) in enumerate(zip(q_len, kv_len, (1, 60, kv_len[2]))):
        dq = c.got(r)[0]
        blind, before = max(n - kv, 0), n - kv + j                    # rows that see nothing, rows in front of the bad key
        assert not dq[:blind].isnan().any() and not dq[:blind].any(), r
        assert dq[:before].isfinite().all(), r
    want, size = c.exact(2)
    for x, w, t in zip(c.got(2), want, c.tolerance(2, size, want)):
        assert ((x - w).abs() <= t).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
def test_rows_without_keys_beside_a_page_outside_the_pool(D, dtype):
    """The place of the keys that are not there holds what an item before has left: here infinities."""
    q_len, kv_len = [128] * 40 + [140], [128] * 40 + [100]
    c = Call(q_len, kv_len, 8, 8, D, dtype, seed=32)
    c.forward()
    c.ctx.check()
    for r in range(40):
        c.k_pages[torch.as_tensor(c.table_host[r][c.table_host[r] >= 0].astype(np.int64), device=G.DEV)] = float("inf")
    c.table[40, 2] = -1                                              # keys 32 .. 47 of the last request
    c.backward()
    with pytest.raises(cb.CascadeError):
        c.ctx.check()
    dq, dk, dv = c.got(40)
    assert not dq[:40].isnan().any() and not dq[:40].any()
    assert dq.isfinite().all() and not dk[32:48].any() and not dv[32:48].any()
