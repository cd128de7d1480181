"""Pages and slots outside the pool: the attention leaves their keys out -- outputs compared with the restatement over the keys
that are left, in every kernel -- and whoever does not see them keeps its results."""
import numpy as np
import pytest
import torch

from paper_2605_07230_b200 import binding as cb
from oracle import paged_oracle as PO
from tests import gpu_util as G
from tests.test_gpu_paged import Case, half_step, i32, make_ctx, run_tables

pytestmark = pytest.mark.gpu


def attention_without(q, k, v, window, sinks, scale, lost):
    """PO.attention over the keys that are not lost: they alone are given to it, row by row."""
    n, kv = q.shape[0], k.shape[0]
    out, lse = np.zeros(q.shape), np.full(q.shape[:2], -np.inf)
    for i in range(n):
        ok = PO.sees(kv - n + i, kv, window, sinks) & ~lost
        out[i: i + 1], lse[i: i + 1] = PO.attention(q[i: i + 1], k[ok], v[ok], 0, 0, scale) if ok.any() else (0.0, -np.inf)
    return out, lse


def check_without(c, bad, window, sinks):
    """bad: request -> table entries that are no pages.  Bounds as in Case.check."""
    out, lse, q = (t.double().cpu().numpy() for t in (c.out, c.lse, c.q))
    at = 0
    for r, (n, kv) in enumerate(zip(c.q_len, c.kv_len)):
        lost = np.isin(np.arange(kv) // c.page, bad.get(r, []))
        ref, ref_lse = attention_without(q[at: at + n], c.k[r], c.v[r], window, sinks, c.scale, lost)
        size, _ = attention_without(q[at: at + n], c.k[r], np.abs(c.v[r]), window, sinks, c.scale, lost)
        w = 2.0 ** -13 + (2.0 ** -8 if c.dtype == "bf16" else 0)
        wrong = ~(np.abs(out[at: at + n] - ref) <= w * size + half_step(ref, c.dtype) + 1e-30)
        assert not wrong.any(), (r, n, kv, np.argwhere(wrong)[:4])
        empty = np.isneginf(ref_lse)
        assert np.array_equal(empty, np.isneginf(lse[at: at + n])), r
        assert (np.abs(lse[at: at + n][~empty] - ref_lse[~empty]) <= 2.0 ** -12 + 2.0 ** -20 * np.abs(ref_lse[~empty])).all(), r
        at += n
    assert (out[at:] == 3).all() and (lse[at:] == 3).all()


def spoil(c, bad):
    for i, (r, entries) in enumerate(bad.items()):
        for j, e in enumerate(entries):
            c.cache.block_table[r, e] = (10 ** 6, -7, c.kp.shape[0], -1)[(i + j) % 4]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,D", [(4, 2, 128), (3, 3, 64)])
@pytest.mark.parametrize("q", [1, 6, 40, 150])
@pytest.mark.parametrize("window,sinks", [(0, 0), (70, 20)])
def test_keys_of_bad_pages_are_left_out(dtype, Hq, Hkv, D, q, window, sinks):
    ctx = make_ctx(dtype, Hq, Hkv, D)
    for page in (8, 16, 128):
        c = Case(dtype, Hq, Hkv, D, page, [q] * 6, [q + 50, q + 51, q + 300, q + 7, q, q + 200], seed=q + page, pad=2)
        last = lambda r: (c.kv_len[r] - 1) // page  # noqa: E731
        bad = {1: [0], 2: [0, last(2) // 2], 3: [last(3)], 4: list(range(last(4) + 1))}      # requests 0 and 5 have their pages
        spoil(c, bad)
        for _ in range(2):
            c.out.fill_(3.0)
            c.lse.fill_(3.0)
            c.run(ctx, window, sinks)
            with pytest.raises(cb.CascadeError) as e:
                ctx.check()
            assert e.value.status == cb.ERR_BAD_PAGE
            check_without(c, bad, window, sinks)
    ctx.close()


def test_neighbours_of_a_bad_page_among_many_items():
    """Several items a CTA, requests with and without bad pages by turns: each its own keys."""
    ctx = make_ctx("bf16", 32, 32, 64)
    c = Case("bf16", 32, 32, 64, 32, [17, 300, 1, 40, 0, 90, 33, 18, 20, 25], [400, 300, 700, 40, 9, 91, 64, 18, 500, 33], seed=5, pad=2)
    bad = {1: [3], 3: [0, 1], 5: [2], 8: [10, 15]}
    spoil(c, bad)
    for _ in range(2):
        c.out.fill_(3.0)
        c.lse.fill_(3.0)
        c.run(ctx)
        with pytest.raises(cb.CascadeError) as e:
            ctx.check()
        assert e.value.status == cb.ERR_BAD_PAGE
        check_without(c, bad, 0, 0)
    ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("q", [1, 40])
def test_requests_beside_one_with_a_bad_length(dtype, q):
    """A length past the bounds leaves that request alone out: its rows stay as they were, the others are right."""
    ctx = make_ctx(dtype, 4, 2, 128)
    c = Case(dtype, 4, 2, 128, 16, [q] * 4, [q + 50] * 4)
    c.kv[1] = 10 ** 6                                            # longer than max_kv and the table
    c.run(ctx)
    with pytest.raises(cb.CascadeError) as e:
        ctx.check()
    assert e.value.status == cb.ERR_BAD_PAGE
    c.check(requests=[0, 2, 3])
    assert (c.out[q: 2 * q] == 3).all() and (c.lse[q: 2 * q] == 3).all()
    ctx.close()
