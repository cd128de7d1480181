"""The paged cache's calls at every count that the header promises."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from oracle import paged_oracle as PO
from paper_2605_07230_b200 import binding as cb
from tests import gpu_util as G
from tests.test_gpu_paged import i32, make_ctx, random_requests, run_tables

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def tables_in_ascending_order():
    """Request counts around the shared memory that a kernel gets unasked, small ones first, in a process of their own (what a
    larger call asked for holds for the smaller ones behind it)."""
    ctx = make_ctx()
    for n_req in (3000, 3022, 3023, 3050, 3071, 3075, 4096):
        rng = np.random.default_rng(n_req)
        new, kv, table, free, count = random_requests(rng, n_req, 8, 3, 20, 0.2)
        n_tok = int(np.maximum(new, 0).sum()) + 1
        ref = PO.tables(new, kv, table, free, count, 8, n_tok)
        got = run_tables(ctx, new, kv, table, free, count, 8, n_tok)
        ctx.check()
        for name in ("table", "free", "kv", "q_begin", "slot", "pos"):
            assert np.array_equal(got[name].cpu().numpy(), ref[name]), (n_req, name)
        assert int(got["count"]) == ref["count"]
    ctx.close()


def test_tables_of_every_request_count():
    r = subprocess.run([sys.executable, "-c", "from tests.test_gpu_paged_counts import tables_in_ascending_order as t; t()"],
                       cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]


def test_fp32_passes_of_more_row_blocks_than_a_grid_has_rows():
    """64 key heads and 32900 new tokens, 65856 blocks of 32 rows; but for the last 40 all rows stand before the first key."""
    H, D, n, kv = 64, 64, 32900, 40
    ctx = make_ctx("f32", H, H, D)
    gen = torch.Generator(device=G.DEV)
    gen.manual_seed(1)
    pool = torch.randn(2, 5, 8, H, D, device=G.DEV, generator=gen)
    cache = cb.PagedCache(pool[0], pool[1], i32([[4, 2, 0, 1, 3]]))
    q = torch.randn(n, H, D, device=G.DEV, generator=gen)
    out, lse = torch.full_like(q, 3.0), torch.full((n, H), 3.0, device=G.DEV)
    cb.cascade_paged_attn(ctx, cache, q, i32([0, n]), i32([kv]), n, kv, out, 0.125, lse=lse)
    ctx.check()
    k, v = (t[torch.tensor([4, 2, 0, 1, 3], device=G.DEV)].view(kv, H, D).double().cpu().numpy() for t in pool)
    ref, ref_lse = PO.attention(q[-kv:].double().cpu().numpy(), k, v, 0, 0, 0.125)
    size, _ = PO.attention(q[-kv:].double().cpu().numpy(), k, np.abs(v), 0, 0, 0.125)
    assert (out[:-kv] == 0).all() and torch.isneginf(lse[:-kv]).all()
    # scores of 64 fp32 products, the weights' and the output's own half steps
    assert (np.abs(out[-kv:].double().cpu().numpy() - ref) <= 2.0 ** -13 * size + 2.0 ** -24 * np.abs(ref)).all()
    assert (np.abs(lse[-kv:].double().cpu().numpy() - ref_lse) <= 2.0 ** -12).all()
    ctx.close()
