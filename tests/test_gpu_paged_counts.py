"""The paged cache's calls at every count that the header promises."""
import os
import subprocess
import sys

import numpy as np
import pytest

from oracle import paged_oracle as PO
from tests.test_gpu_paged import make_ctx, random_requests, run_tables

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def tables_in_ascending_order():
    """Request counts around the shared memory that a kernel gets unasked, small ones first, in a process of their own (what a
    larger call asked for holds for the smaller ones behind it)."""
    ctx = make_ctx()
    for n_req in (3000, 3022, 3023, 3050, 3071, 3072, 4096):
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
