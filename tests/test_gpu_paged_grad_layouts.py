"""GPU: the paged attention's gradient over pools and tables of other layouts: keys and values in one pool, tables that are slices,
pages shared by requests, queries behind a first row, odd and large pages, offsets past 32 bits, lengths that change between replays."""
import numpy as np
import pytest
import torch

from paper_2605_07230_b200 import binding as cb
from tests import gpu_util as G
from tests.test_gpu_paged_grad import DT, Call, i32

pytestmark = pytest.mark.gpu

TYPES = pytest.mark.parametrize("dtype", ["bf16", "f32"])


def check_requests(c, requests=None):
    for r in requests if requests is not None else range(len(c.q_len)):
        want, size = c.exact(r)
        for name, x, w, t in zip(("dq", "dk", "dv"), c.got(r), want, c.tolerance(r, size, want)):
            assert ((x - w).abs() <= t).all(), (r, name)


@TYPES
@pytest.mark.parametrize("D", [64, 128])
def test_keys_and_values_in_one_pool_and_a_slice_of_a_table(D, dtype):
    c = Call([60, 1, 200], [75, 130, 200], 6, 2, D, dtype, page=24, window=90, sinks=5, seed=51, pad=1)
    pool = torch.full((c.k_pages.shape[0], 3, 24, 2, D), float("nan"), device=G.DEV, dtype=DT[dtype])
    pool[:, 0], pool[:, 2] = c.k_pages, c.v_pages
    c.k_pages, c.v_pages = pool[:, 0], pool[:, 2]
    wide = torch.full((5, c.table.shape[1] + 9), 2**31 - 1, device=G.DEV, dtype=torch.int32)
    wide[1:4, 2: 2 + c.table.shape[1]] = c.table
    c.table = wide[1:4, 2: 2 + c.table.shape[1]]
    c.cache = cb.PagedCache(c.k_pages, c.v_pages, c.table)
    c.run().check()


@TYPES
def test_pages_shared_by_requests_have_gradients_of_their_own(dtype):
    c = Call([30, 50, 7], [110, 130, 87], 4, 2, 64, dtype, seed=52)
    c.table_host[1:, :5] = c.table_host[0, :5]                       # eighty keys in front of all three
    c.table.copy_(i32(c.table_host))
    c.run().check()


@TYPES
def test_queries_behind_a_first_row(dtype):
    c = Call([20, 130], [40, 130], 4, 4, 64, dtype, seed=53, pad=9)
    c.q_begin += 5
    c.run()
    check_requests(c)
    assert c.dq[:5].isnan().all() and c.dq[155:].isnan().all()


@TYPES
@pytest.mark.parametrize("page", [40, 136, 384, 1000])
def test_page_sizes_around_and_above_a_tile(page, dtype):
    Call([50, 3, 140], [page + 30, 2 * page + 7, 140], 4, 2, 64, dtype, page=page, window=300, sinks=9, seed=page, pad=1).run().check()


@TYPES
@pytest.mark.parametrize("q_len,kv_len", [([100], [100]), ([1, 300], [70, 420])])
def test_pools_whose_offsets_pass_32_bits(q_len, kv_len, dtype):
    """70000 pages of 16 rows, 16 heads of 128: 2.3e9 elements each."""
    c = Call(q_len, kv_len, 16, 16, 128, dtype, seed=54)
    few, many = c.k_pages.shape[0], 70000
    at = np.linspace(0, many - 1, few).astype(np.int64)              # page p of the small pool -> page at[p]
    big = [torch.empty((many, 16, 16, 128), device=G.DEV, dtype=DT[dtype]) for _ in range(2)]
    for to, small in zip(big, (c.k_pages, c.v_pages)):
        to[torch.as_tensor(at, device=G.DEV)] = small
    c.k_pages, c.v_pages = big
    c.table_host = np.where(c.table_host >= 0, at[c.table_host], -1).astype(np.int32)
    c.table.copy_(i32(c.table_host))
    c.cache = cb.PagedCache(c.k_pages, c.v_pages, c.table)
    c.run().check()


@TYPES
def test_lengths_that_change_between_replays(dtype):
    """One graph for batches of several shapes within its bounds."""
    c = Call([40, 150, 10], [60, 150, 90], 4, 2, 64, dtype, seed=55, pad=100)
    c.max_q, c.max_kv = 290, 300
    c.forward()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.backward()
    for q_len, kv_len in (([40, 150, 10], [60, 150, 90]), ([0, 1, 37], [3, 20, 40]), ([33, 0, 3], [33, 0, 10]), ([1, 1, 1], [1, 144, 90])):
        c.q_len, c.kv_len_host = q_len, kv_len
        c.q_begin.copy_(i32(np.concatenate([[0], np.cumsum(q_len)])))
        c.kv_len.copy_(i32(kv_len))
        for t in (c.dq, c.dk, c.dv):
            t.fill_(float("nan"))
        c.forward()
        graph.replay()
        c.ctx.check()
        c.check()
