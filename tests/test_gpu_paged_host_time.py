"""A server's passes differ in their number of tokens: a call after thousands of others costs the host no more than the first."""
import time

import numpy as np
import pytest
import torch

from paper_2605_07230_b200 import binding as cb
from tests import gpu_util as G
from tests.test_gpu_paged import i32, make_ctx

pytestmark = pytest.mark.gpu


def test_host_time_of_a_chunk_does_not_grow_with_the_passes_before_it():
    ctx = make_ctx("bf16", 2, 2, 64)
    pool = torch.zeros(2, 8, 16, 2, 64, dtype=torch.bfloat16, device=G.DEV)
    cache = cb.PagedCache(pool[0], pool[1], i32([[0, 1, 2, 3, 4]]))
    q = torch.zeros(4000, 2, 64, dtype=torch.bfloat16, device=G.DEV)
    out = torch.zeros_like(q)
    begin, kv = i32([0, 20]), i32([50])

    def call(n):
        cb.cascade_paged_attn(ctx, cache, q[:n], begin, kv, 20, 80, out[:n], 0.125)

    def median_us(n):
        times = []
        for i in range(200):
            t = time.perf_counter()
            call(n)
            times.append(time.perf_counter() - t)
            if i % 50 == 49:
                torch.cuda.synchronize()
        return 1e6 * float(np.median(times))

    call(30)
    first = median_us(30)
    for n in range(40, 3540):
        call(n)
    torch.cuda.synchronize()
    last = median_us(3600)
    ctx.check()
    print(f"host time of a call: {first:.1f} us, after 3500 lengths {last:.1f} us")
    assert last < 2 * first + 5, (first, last)
    ctx.close()
