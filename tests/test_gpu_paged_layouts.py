"""The paged calls at the widest groups of query heads, at page sizes around and above a key tile, and in pools whose offsets
pass 32 bits."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as PO
from paper_2605_07230_b200 import binding as cb
from tests import gpu_util as G
from tests.test_gpu_paged import Case, DT, half_step, i32, make_ctx

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,D", [(128, 1, 64), (127, 1, 128), (130, 2, 64), (200, 2, 128), (17, 1, 64)])
def test_wide_groups(dtype, Hq, Hkv, D):
    ctx = make_ctx(dtype, Hq, Hkv, D)
    for q, kv in (([1, 1], [33, 140]), ([3, 1, 2], [3, 129, 200])):
        c = Case(dtype, Hq, Hkv, D, 16, q, kv, seed=Hq, pad=1)
        c.q[sum(q):] = float("nan")                              # rows behind the last token do not matter
        c.run(ctx)
        ctx.check()
        c.check()
    ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [24, 40, 136, 384, 1024])
@pytest.mark.parametrize("side_by_side", [True, False])
def test_page_sizes(dtype, page, side_by_side):
    ctx = make_ctx(dtype, 4, 2, 64)
    for q, kv in (([1, 1, 1], [page, page + 1, 2 * page + 7]), ([40, 9], [page + 30, 3 * page])):
        for window, sinks in ((0, 0), (50, 3)):
            c = Case(dtype, 4, 2, 64, page, q, kv, seed=page, pad=1, side_by_side=side_by_side)
            c.run(ctx, window, sinks)
            ctx.check()
            c.check(window, sinks)
            with_lse = c.out.clone()
            c.out.fill_(3.0)
            c.run(ctx, window, sinks, lse=False)
            ctx.check()
            assert torch.equal(c.out, with_lse)
    ctx.close()


@pytest.mark.parametrize("dtype,n_pages,q", [("bf16", 70000, 1), ("bf16", 70000, 60), ("f32", 70000, 1), ("f32", 70000, 60)])
def test_pools_whose_offsets_pass_32_bits(dtype, n_pages, q):
    """70000 pages of 16 rows, 16 heads of 128: 2.3e9 elements each; keys on both sides of element 2^31, written and read."""
    H, D, page, kv = 16, 128, 16, 100
    ctx = make_ctx(dtype, H, H, D)
    rng = np.random.default_rng(q)
    k_pages, v_pages = (torch.empty(n_pages, page, H, D, dtype=DT[dtype], device=G.DEV) for _ in range(2))
    last, edge = n_pages - 1, 2 ** 31 // (page * H * D)
    table = np.array([[last, 3, edge, edge - 1, last - 7, 0, edge + 1]])
    cache = cb.PagedCache(k_pages, v_pages, i32(table))
    x = torch.from_numpy(rng.normal(size=(3, kv, H, D)).astype(np.float32)).to(DT[dtype]).to(G.DEV)
    where = np.arange(kv)
    slot = table[0][where // page] * page + where % page
    cb.cascade_paged_append(ctx, cache, x[0], x[1], i32(slot), i32(where))
    at = torch.from_numpy(table[0][where // page]).to(G.DEV), torch.from_numpy(where % page).to(G.DEV)
    assert torch.equal(k_pages[at], x[0]) and torch.equal(v_pages[at], x[1])
    out, lse = torch.zeros(q, H, D, dtype=DT[dtype], device=G.DEV), torch.zeros(q, H, device=G.DEV)
    cb.cascade_paged_attn(ctx, cache, x[2, :q], i32([0, q]), i32([kv]), q, kv, out, D ** -0.5, lse=lse)
    ctx.check()
    qq, k, v = (t.double().cpu().numpy() for t in (x[2, :q], x[0], x[1]))
    ref, ref_lse = PO.attention(qq, k, v, 0, 0, D ** -0.5)
    size, _ = PO.attention(qq, k, np.abs(v), 0, 0, D ** -0.5)
    tol = (2.0 ** -13 + (2.0 ** -8 if dtype == "bf16" else 0)) * size + half_step(ref, dtype)
    assert (np.abs(out.double().cpu().numpy() - ref) <= tol).all()
    assert (np.abs(lse.double().cpu().numpy() - ref_lse) <= 2.0 ** -12 + 2.0 ** -20 * np.abs(ref_lse)).all()
    ctx.close()
