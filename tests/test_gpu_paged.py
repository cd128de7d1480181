"""GPU parity of the paged cache's calls against their 64-bit restatements: block tables, slots and free pages exact;
rotated rows within half a step of their type; attention within bounds that count its roundings."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from oracle import paged_oracle as PO
from paper_2605_07230_b200 import binding as cb
from tests import gpu_util as G

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def make_ctx(dtype="bf16", Hq=4, Hkv=4, D=64, V=64):
    return cb.Context(cb.BF16 if dtype == "bf16" else cb.F32, 1, 1, 64, 64, Hq, Hkv, D, V)


def i32(x):
    return torch.as_tensor(np.asarray(x, np.int32), device=G.DEV)


# ---- tables ---------------------------------------------------------------------------------------------------------


def run_tables(ctx, new, kv, table, free, count, page, n_tok, in_place=True):
    n_pages = len(free)
    d = dict(new=i32(new), kv=i32(kv), table=i32(table), free=i32(free), count=i32([count]), q_begin=i32([-9] * (len(new) + 1)),
             slot=i32([-9] * n_tok), pos=i32([-9] * n_tok))
    kv_out = d["kv"] if in_place else i32([-9] * len(new))
    count_out = d["count"] if in_place else i32([-9])
    cb.cascade_paged_tables(ctx, page, n_pages, d["new"], d["kv"], d["table"], d["free"], d["count"], kv_out, count_out,
                            d["q_begin"], d["slot"], d["pos"])
    torch.cuda.synchronize()
    return dict(table=d["table"], free=d["free"], kv=kv_out, q_begin=d["q_begin"], slot=d["slot"], pos=d["pos"], count=count_out)


def random_requests(rng, n_req, page, q_hi, kv_hi, done, spare=3):
    kv = rng.integers(0, kv_hi + 1, n_req)
    new = np.where(rng.random(n_req) < done, -1, rng.integers(0, q_hi + 1, n_req))
    pages = lambda n: -(-n // page)  # noqa: E731
    width = int(pages(kv + np.maximum(new, 0)).max()) + 1
    n_pages = int(pages(kv).sum() + (pages(kv + np.maximum(new, 0)) - pages(kv)).sum()) + spare
    ids = rng.permutation(n_pages)
    table, at = np.full((n_req, width), -1), 0
    for r in range(n_req):
        table[r, : pages(kv[r])] = ids[at: at + pages(kv[r])]
        at += pages(kv[r])
    free = np.full(n_pages, -5)
    free[: n_pages - at] = ids[at:]
    return new, kv, table, free, n_pages - at


@pytest.mark.parametrize("n_req,page,q_hi,kv_hi,done,pad", [(1, 8, 1, 0, 0.0, 0), (2, 16, 1, 400, 0.0, 3), (7, 8, 30, 50, 0.3, 1),
                                                            (65, 16, 3, 300, 0.5, 0), (300, 48, 200, 500, 0.1, 77),
                                                            (1025, 16, 40, 90, 0.2, 5), (4096, 8, 9, 20, 0.3, 2)])
@pytest.mark.parametrize("in_place", [True, False])
def test_tables(n_req, page, q_hi, kv_hi, done, pad, in_place):
    rng = np.random.default_rng(n_req)
    ctx = make_ctx()
    new, kv, table, free, count = random_requests(rng, n_req, page, q_hi, kv_hi, done)
    n_tok = int(np.maximum(new, 0).sum()) + pad
    ref = PO.tables(new, kv, table, free, count, page, n_tok)
    got = run_tables(ctx, new, kv, table, free, count, page, n_tok, in_place)
    ctx.check()
    for name in ("table", "free", "kv", "q_begin", "slot", "pos"):
        assert np.array_equal(got[name].cpu().numpy(), ref[name]), name
    assert int(got["count"]) == ref["count"]
    ctx.close()


@pytest.mark.parametrize("what", ["pool", "rows", "width", "length", "count", "give back"])
def test_tables_take_nothing_when_something_does_not_fit(what):
    new, kv, count, n_tok = [4, -1, 8], [5, 9, 0], 2, 14
    table, free = [[7, -1, -1], [4, 2, -1], [-1, -1, -1]], [3, 6, 0, 0, 0, 0, 0, 0]
    if what == "pool":
        new, count = [12, -1, 24], 0
    if what == "rows":
        n_tok = 11
    if what == "width":
        new = [20, -1, 8]
    if what == "length":
        kv = [-5, 9, 0]
    if what == "count":
        count = 9
    if what == "give back":
        count = 7
    assert PO.tables(new, kv, table, free, count, 8, n_tok) is None
    ctx = make_ctx()
    for in_place in (True, False):
        got = run_tables(ctx, new, kv, table, free, count, 8, n_tok, in_place)
        with pytest.raises(cb.CascadeError) as e:
            ctx.check()
        assert e.value.status == cb.ERR_OVERFLOW
        assert got["table"].tolist() == table and got["free"].tolist() == free and got["kv"].tolist() == kv
        assert int(got["count"]) == count and set(got["q_begin"].tolist()) == {0} and set(got["slot"].tolist()) == {-1}
        assert set(got["pos"].tolist()) == {-1}
    ctx.check()          # the word was cleared
    ctx.close()


def test_tables_of_lengths_at_the_end_of_32_bits():
    P, top = 1 << 28, 2**31 - 1                     # ten entries of a row reach past 2^31 tokens, the pool does not
    ctx = make_ctx()
    for new, kv in (([10], [top]), ([top], [top]), ([1], [top])):
        got = run_tables(ctx, new, kv, [[0, 1, 2, 3, 4, 5, 6, 7, -1, -1]], [0] * 7, 0, P, 16)
        with pytest.raises(cb.CascadeError) as e:
            ctx.check()
        assert e.value.status == cb.ERR_OVERFLOW
        assert got["kv"].tolist() == kv and set(got["slot"].tolist()) == {-1}
    got = run_tables(ctx, [1], [6 * P + P - 2], [[3, 1, 2, 0, 4, 5, 6, -1]], [0] * 7, 0, P, 2)
    ctx.check()
    assert got["slot"].tolist() == [6 * P + P - 2, -1] and got["pos"].tolist() == [7 * P - 2, -1]
    ctx.close()


def test_tables_without_rows_and_with_a_bad_page():
    ctx = make_ctx()
    got = run_tables(ctx, [0, -1], [9, 8], [[1, 0], [2, -1]], [-1, -1, -1, -1], 0, 8, 0)
    assert got["kv"].tolist() == [9, 0] and int(got["count"]) == 1 and got["free"].tolist()[0] == 2
    ctx.check()
    got = run_tables(ctx, [2, 1], [9, 3], [[1, 99], [2, -1]], [0, 0, 0, 0], 1, 8, 4)
    assert got["slot"].tolist() == [-1, -1, 19, -1]
    with pytest.raises(cb.CascadeError) as e:
        ctx.check()
    assert e.value.status == cb.ERR_BAD_PAGE
    ctx.close()


# ---- append ---------------------------------------------------------------------------------------------------------


def half_step(x, dtype):
    return np.abs(x) * (torch.finfo(DT[dtype]).eps / 2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,Hq,Hkv,D,page,far", [(1, 4, 4, 64, 8, 0), (7, 8, 2, 128, 16, 3000), (33, 5, 1, 64, 48, 100000),
                                                 (130, 32, 32, 128, 16, 2400)])
def test_append(dtype, n, Hq, Hkv, D, page, far):
    rng = np.random.default_rng(n)
    ctx = make_ctx(dtype, Hq, Hkv, D)
    n_pages = -(-n // page) + 2
    pool = torch.full((n_pages, 2, page, Hkv, D), 7.0, dtype=DT[dtype], device=G.DEV)   # keys and values of a page side by side
    cache = cb.PagedCache(pool[:, 0], pool[:, 1], i32([[0]]))
    qkv = torch.from_numpy(rng.normal(size=(n, (Hq + 2 * Hkv) * D)).astype(np.float32)).to(G.DEV).to(DT[dtype])
    q, k, v = (t.unflatten(1, (-1, D)) for t in qkv.split([Hq * D, Hkv * D, Hkv * D], 1))
    slot = rng.permutation(n_pages * page)[:n]
    pos = rng.integers(0, far + 1, n)
    slot[n // 2] = -1 if n > 1 else slot[0]
    q_out = torch.full((n, Hq, D), 5.0, dtype=DT[dtype], device=G.DEV)
    before = qkv.clone()
    cb.cascade_paged_append(ctx, cache, k, v, i32(slot), i32(pos), 10000.0, q, q_out)
    torch.cuda.synchronize()
    ctx.check()
    assert torch.equal(before, qkv) and ctx.last_launch_count == 1
    live = slot >= 0
    kk, vv = pool[:, 0].reshape(-1, Hkv, D), pool[:, 1].reshape(-1, Hkv, D)
    f = lambda t: t.double().cpu().numpy()  # noqa: E731
    # a rotated element: two fp32 products and a sum of angles good to 2^-23, then the type's own half step
    tol = lambda x, ref: half_step(ref, dtype) + 2.0 ** -21 * np.abs(f(x)).max()  # noqa: E731
    for got, x in ((f(kk)[slot[live]], k), (f(q_out)[live], q)):
        ref = PO.rotate(f(x)[live], pos[live], 10000.0)
        assert (np.abs(got - ref) <= tol(x, ref)).all()
    assert np.array_equal(f(vv)[slot[live]], f(v)[live])
    rest = np.setdiff1d(np.arange(n_pages * page), slot)
    assert (f(kk)[rest] == 7).all() and (f(vv)[rest] == 7).all() and (f(q_out)[~live] == 5).all()
    # without rotation and without queries: copies; with queries in place
    cb.cascade_paged_append(ctx, cache, k, v, i32(slot), i32(pos))
    assert np.array_equal(f(pool[:, 0].reshape(-1, Hkv, D))[slot[live]], f(k)[live])
    cb.cascade_paged_append(ctx, cache, k, v, i32(slot), i32(pos), 10000.0, q, q)
    assert np.array_equal(f(q)[live], f(q_out)[live])
    ctx.close()


def test_append_leaves_bad_slots_out():
    ctx = make_ctx("bf16", 4, 2, 64)
    pool = torch.zeros(2, 8, 2, 64, dtype=torch.bfloat16, device=G.DEV)
    cache = cb.PagedCache(pool, pool.clone(), i32([[0]]))
    k = torch.ones(3, 2, 64, dtype=torch.bfloat16, device=G.DEV)
    cb.cascade_paged_append(ctx, cache, k, k, i32([3, 16, 2 ** 31 - 1]), i32([0, 0, 0]))
    torch.cuda.synchronize()
    assert float(pool.float().sum()) == 128 and float(cache.v_pages.float().sum()) == 128
    with pytest.raises(cb.CascadeError) as e:
        ctx.check()
    assert e.value.status == cb.ERR_BAD_PAGE
    ctx.close()


# ---- attention ------------------------------------------------------------------------------------------------------


class Case:
    """Requests over a shuffled pool whose unused rows and pages hold NaN."""

    def __init__(self, dtype, Hq, Hkv, D, page, q_len, kv_len, seed=0, pad=0, scale=1.0, extra_width=1, side_by_side=False):
        rng = np.random.default_rng(seed)
        self.dims = (Hq, Hkv, D)
        self.dtype, self.page, self.q_len, self.kv_len = dtype, page, list(q_len), list(kv_len)
        n_req = len(q_len)
        counts = [-(-n // page) for n in kv_len]
        n_pages = sum(counts) + 2
        shape = (n_pages, 2, page, Hkv, D) if side_by_side else (2, n_pages, page, Hkv, D)
        pool = torch.full(shape, float("nan"), dtype=DT[dtype], device=G.DEV)
        self.kp, self.vp = (pool[:, 0], pool[:, 1]) if side_by_side else (pool[0], pool[1])
        ids = rng.permutation(n_pages)
        width = max(max(counts), 1) + extra_width
        table, at = np.full((n_req, width), 10 ** 9), 0
        self.k, self.v = [], []
        for r, n in enumerate(kv_len):
            table[r, : counts[r]] = ids[at: at + counts[r]]
            at += counts[r]
            for pool_t, keep in ((self.kp, self.k), (self.vp, self.v)):
                x = torch.from_numpy(rng.normal(size=(n, Hkv, D)).astype(np.float32)).to(DT[dtype])
                keep.append(x.double().numpy())
                where = np.arange(n)
                pool_t[torch.from_numpy(table[r][where // page]).to(G.DEV), torch.from_numpy(where % page).to(G.DEV)] = x.to(G.DEV)
        N = sum(q_len) + pad
        q = torch.from_numpy((scale * rng.normal(size=(max(N, 1), Hq + 1, D))).astype(np.float32)).to(DT[dtype]).to(G.DEV)
        self.q = q[:, :Hq]                                    # rows lie apart
        self.table, self.cache = table, cb.PagedCache(self.kp, self.vp, i32(table))
        self.q_begin, self.kv = i32(np.concatenate([[0], np.cumsum(q_len)])), i32(kv_len)
        self.out = torch.full((max(N, 1), Hq, D), 3.0, dtype=DT[dtype], device=G.DEV)
        self.lse = torch.full((max(N, 1), Hq), 3.0, device=G.DEV)
        self.scale = 1.0 / math.sqrt(D)

    def run(self, ctx, window=0, sinks=0, max_q=None, max_kv=None, lse=True):
        cb.cascade_paged_attn(ctx, self.cache, self.q, self.q_begin, self.kv, max_q or max(max(self.q_len), 1),
                              max(self.kv_len) if max_kv is None else max_kv, self.out, self.scale, window=window, sinks=sinks,
                              lse=self.lse if lse else None)
        torch.cuda.synchronize()

    def check(self, window=0, sinks=0, requests=None):
        Hq, Hkv, D = self.dims
        at = 0
        out, lse = self.out.double().cpu().numpy(), self.lse.double().cpu().numpy()
        q = self.q.double().cpu().numpy()
        for r, (n, kv) in enumerate(zip(self.q_len, self.kv_len)):
            if requests is None or r in requests:
                ref, ref_lse = PO.attention(q[at: at + n], self.k[r], self.v[r], window, sinks, self.scale)
                size, _ = PO.attention(q[at: at + n], self.k[r], np.abs(self.v[r]), window, sinks, self.scale)
                # fp32 scores of D products: each weight is off by at most about D 2^-24 sum |q k| scale, under 2^-13 for
                # these inputs; bf16: the weights' own rounding (half a step of the weighted |v|) and the output's
                w = 2.0 ** -13 + (2.0 ** -8 if self.dtype == "bf16" else 0)
                tol = w * size + half_step(ref, self.dtype) + 1e-30
                got = out[at: at + n]
                bad = ~(np.abs(got - ref) <= tol)
                assert not bad.any(), (r, n, kv, np.argwhere(bad)[:4], np.abs(got - ref).max())
                empty = np.isneginf(ref_lse)
                assert np.array_equal(empty, np.isneginf(lse[at: at + n]))
                assert (np.abs(lse[at: at + n][~empty] - ref_lse[~empty]) <= 2.0 ** -12 + 2.0 ** -20 * np.abs(ref_lse[~empty])).all()
            at += n
        assert (out[at:] == 3).all() and (lse[at:] == 3).all()           # rows behind the last request


HEADS = [(4, 4, 64), (4, 4, 128), (8, 2, 128), (10, 2, 64), (16, 1, 128), (7, 1, 64), (40, 1, 128)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,D", HEADS)
def test_single_tokens(dtype, Hq, Hkv, D):
    ctx = make_ctx(dtype, Hq, Hkv, D)
    for page, kv in ((16, [1, 2, 7, 8, 9, 15, 16, 17, 31, 33, 64, 65]), (8, [130, 127, 1, 200]), (48, [97, 500, 48, 49])):
        c = Case(dtype, Hq, Hkv, D, page, [1] * len(kv), kv, seed=page, pad=2)
        c.run(ctx)
        ctx.check()
        c.check()
    ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,D", HEADS)
def test_chunks(dtype, Hq, Hkv, D):
    ctx = make_ctx(dtype, Hq, Hkv, D)
    for page, q, kv in ((16, [5, 1, 17, 3, 8], [5, 40, 33, 128, 129]), (8, [2, 9, 1], [200, 9, 1]), (64, [40, 63, 1], [290, 64, 65])):
        c = Case(dtype, Hq, Hkv, D, page, q, kv, seed=page, pad=3)
        c.run(ctx)
        ctx.check()
        c.check()
    ctx.close()


@pytest.mark.parametrize("Hq,Hkv,D", [(2, 2, 128), (4, 1, 128), (2, 2, 64), (3, 1, 64)])
def test_prompts(Hq, Hkv, D):
    """Several row blocks and key tiles, a first chunk beside chunks behind a prefix, requests without new tokens."""
    ctx = make_ctx("bf16", Hq, Hkv, D)
    for page, q, kv in ((16, [300, 0, 129, 1], [300, 20, 400, 391]), (32, [128, 257], [128, 257]), (24, [255], [777])):
        c = Case("bf16", Hq, Hkv, D, page, q, kv, seed=page, pad=5, side_by_side=True)
        c.run(ctx)
        ctx.check()
        c.check()
    ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,D", [(4, 4, 64), (8, 2, 128)])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (16, 4), (50, 0), (100, 17), (130, 129), (1000, 4), (64, 10 ** 6)])
def test_window_and_sinks(dtype, Hq, Hkv, D, window, sinks):
    ctx = make_ctx(dtype, Hq, Hkv, D)
    for q, kv in (([1, 1, 1], [400, 17, 1]), ([9, 30, 1], [300, 30, 390]), ([140, 2], [500, 64])):
        c = Case(dtype, Hq, Hkv, D, 16, q, kv, seed=window)
        c.run(ctx, window, sinks)
        ctx.check()
        c.check(window, sinks)
    ctx.close()


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 64)])
@pytest.mark.parametrize("q", [1, 3, 70])
def test_rows_that_see_nothing(dtype, D, q):
    """Fewer keys than new tokens: the first rows stand before the first key.  No keys, no tokens."""
    ctx = make_ctx(dtype, 4, 4, D)
    c = Case(dtype, 4, 4, D, 16, [q, q, q, 0], [0, max(q - 2, 0), q, 5], pad=1)
    c.run(ctx)
    ctx.check()
    c.check()
    c = Case(dtype, 4, 4, D, 16, [q, 0], [0, 0])
    c.run(ctx)
    c.check()
    ctx.close()


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 128)])
@pytest.mark.parametrize("q,kv,window,sinks", [(1, 300, 40, 3), (6, 70, 0, 0), (150, 300, 40, 3), (150, 150, 0, 0)])
def test_what_is_not_seen_does_not_matter(dtype, D, q, kv, window, sinks):
    """NaN and infinite keys and values at places that a row does not see leave it as it is; rows that see them are NaN."""
    Hq = Hkv = 2
    ctx = make_ctx(dtype, Hq, Hkv, D)
    c = Case(dtype, Hq, Hkv, D, 16, [q], [kv], scale=1.0)
    c.run(ctx, window, sinks)
    c.check(window, sinks)
    clean = c.out.clone()
    for x in (kv - 1, kv - 1 - q // 2, 60, 5, 0):
        if x < 0:
            continue
        for pool, bad in ((c.kp, float("nan")), (c.vp, float("inf")), (c.vp, float("nan"))):
            page, row = int(c.table[0, x // 16]), x % 16
            keep = pool[page, row].clone()
            pool[page, row] = bad
            c.run(ctx, window, sinks)
            pool[page, row] = keep
            sees = np.array([PO.sees(kv - q + i, kv, window, sinks)[x] for i in range(q)])
            got = c.out.float().cpu().numpy()
            blind = got[~sees]
            # a row that meets a non-finite neighbour may be summed in another order: half a step of bf16 weights apart
            assert np.isfinite(blind).all()
            ref, _ = PO.attention(c.q.double().cpu().numpy()[~sees], c.k[0], c.v[0], window, sinks, c.scale) if q == 1 else (None, None)
            assert np.abs(blind - clean.float().cpu().numpy()[~sees]).max(initial=0) <= 2.0 ** -6 * max(1.0, float(clean.abs().max()))
            assert not np.isfinite(got[sees]).all(-1).any()
    ctx.check()
    ctx.close()


def test_peaked_and_flat_scores():
    """Scores of a few hundred in both directions, rising and falling along the keys, and all alike."""
    for D, q in ((128, [1, 40]), (64, [2, 200])):
        ctx = make_ctx("bf16", 2, 2, D)
        for scale in (0.0, 30.0):
            c = Case("bf16", 2, 2, D, 16, q, [400, 450], scale=scale, seed=5)
            if scale > 0:       # integer queries and keys: scores are exact, so only the weights' roundings remain
                c.q.copy_(torch.round(c.q))
                for r, kv in enumerate(c.kv_len):
                    k = np.round(c.k[r] * 4 * np.linspace(0.1, 1, kv)[:, None, None])
                    c.k[r] = k
                    where = np.arange(kv)
                    c.kp[torch.from_numpy(c.table[r][where // 16]).to(G.DEV), torch.from_numpy(where % 16).to(G.DEV)] = \
                        torch.from_numpy(k).to(G.DEV).to(torch.bfloat16)
            c.run(ctx)
            ctx.check()
            Hq, _, _ = c.dims
            at = 0
            for r, n in enumerate(c.q_len):
                qq = c.q[at: at + n].double().cpu().numpy()
                ref, _ = PO.attention(qq, c.k[r], c.v[r], 0, 0, c.scale)
                size, _ = PO.attention(qq, c.k[r], np.abs(c.v[r]), 0, 0, c.scale)
                # fp32 exponents: a score of s leaves |s| 2^-22 of relative error in its weight
                most = np.abs(np.einsum("nhd,khd->nhk", qq, c.k[r])).max() * c.scale
                tol = (2.0 ** -8 + 2.0 ** -13 + most * 2.0 ** -21) * size + half_step(ref, "bf16")
                assert (np.abs(c.out[at: at + n].double().cpu().numpy() - ref) <= tol).all()
                at += n
        ctx.close()


def test_bad_pages_and_lengths_are_left_out():
    ctx = make_ctx("bf16", 4, 2, 128)
    for q in (1, 40):
        c = Case("bf16", 4, 2, 128, 16, [q] * 4, [q + 50] * 4)
        table = c.cache.block_table
        table[1, 1] = 10 ** 6
        table[2, 0] = -7
        c.run(ctx)
        with pytest.raises(cb.CascadeError) as e:
            ctx.check()
        assert e.value.status == cb.ERR_BAD_PAGE
        c.lse[:] = 3.0
        c.out[:] = 3.0
        c = Case("bf16", 4, 2, 128, 16, [q] * 4, [q + 50] * 4)
        c.kv[1] = 10 ** 6            # longer than max_kv and the table
        c.q_begin[4] = 4 * q + 100   # beyond the rows there are
        c.run(ctx)
        with pytest.raises(cb.CascadeError):
            ctx.check()
        c.kv_len[1] = q + 50
        got = c.out.float().cpu().numpy()
        assert (got[q: 2 * q] == 3).all() and (got[3 * q:] == 3).all() and (got[:q] != 3).any() and (got[2 * q: 3 * q] != 3).any()
    ctx.close()


def test_graph_replay_with_other_lengths():
    """Recorded once with host bounds, replayed after the device-resident lengths, tables and inputs have changed."""
    ctx = make_ctx("bf16", 4, 4, 128)
    c = Case("bf16", 4, 4, 128, 16, [7, 33], [200, 150], pad=4, extra_width=5)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        c.run(ctx, max_q=40, max_kv=300)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=st):
        cb.cascade_paged_attn(ctx, c.cache, c.q, c.q_begin, c.kv, 40, 300, c.out, c.scale, lse=c.lse)
    d = Case("bf16", 4, 4, 128, 16, [37, 3], [120, 230], seed=9, pad=4)
    for a, b in ((c.q, d.q), (c.q_begin, d.q_begin), (c.kv, d.kv)):
        a.copy_(b)
    n = min(c.table.shape[1], d.table.shape[1])
    pages = min(c.kp.shape[0], d.kp.shape[0])
    assert d.kp.shape[0] <= c.kp.shape[0] and n >= 15
    c.kp[:pages], c.vp[:pages] = d.kp[:pages], d.vp[:pages]
    c.cache.block_table[:, :n] = d.cache.block_table[:, :n]
    c.out.fill_(3.0)
    c.lse.fill_(3.0)
    g.replay()
    torch.cuda.synchronize()
    ctx.check()
    d.out, d.lse = c.out, c.lse
    d.check()
    ctx.close()


def test_prompt_into_the_dense_cache_then_tree():
    """The calls together, as a server would run them: pages for two prompts, their keys and values appended and attended to
    in two passes, the pool being the dense prefix cache that the tree attention then reads; a token drawn at the end."""
    Hq = Hkv = 4
    D, T, cap, page = 128, 15, 256, 16
    from paper_2605_07230_b200 import synth
    parent = synth.complete_tree(2, 3)
    ctx = cb.Context(cb.BF16, 1, T, cap, 512, Hq, Hkv, D, 1024)
    tree = cb.Tree(ctx, parent)
    rng = np.random.default_rng(4)
    bf = lambda x: torch.from_numpy(x.astype(np.float32)).to(G.DEV).to(torch.bfloat16)  # noqa: E731
    kc, vc = (torch.full((2, cap, Hkv, D), float("nan"), dtype=torch.bfloat16, device=G.DEV) for _ in range(2))
    per = cap // page
    pool = [t.view(2 * per, page, Hkv, D) for t in (kc, vc)]
    table = torch.arange(2 * per, dtype=torch.int32, device=G.DEV).view(2, per)          # the dense layout's own table
    cache = cb.PagedCache(pool[0], pool[1], table)
    kv, q_begin, count = i32([0, 0]), i32([0, 0, 0]), i32([2 * per])
    # the free stack that hands out exactly these pages: request by request
    lens = ([90, 37], [41, 55])
    keys, vals, total = [[], []], [[], []], [0, 0]
    for chunk in lens:
        n = sum(chunk)
        x = bf(rng.normal(size=(n + 3, (Hq + 2 * Hkv) * D)))                            # three padded rows
        q, k, v = (t.unflatten(1, (-1, D)) for t in x.split([Hq * D, Hkv * D, Hkv * D], 1))
        slot, pos = i32([-9] * (n + 3)), i32([-9] * (n + 3))
        need = [-(-(t + c) // page) - -(-t // page) for t, c in zip(total, chunk)]
        order = [r * per + -(-total[r] // page) + j for r in range(2) for j in range(need[r])]
        free = i32(order[::-1] + [0] * (2 * per - len(order)))
        cnt = i32([len(order)])
        cb.cascade_paged_tables(ctx, page, 2 * per, i32(chunk), kv, table, free, cnt, kv, cnt, q_begin, slot, pos)
        qr = torch.empty_like(q)
        cb.cascade_paged_append(ctx, cache, k, v, slot, pos, 10000.0, q, qr)
        out = torch.full((n + 3, Hq, D), 3.0, dtype=torch.bfloat16, device=G.DEV)
        cb.cascade_paged_attn(ctx, cache, qr, q_begin, kv, max(chunk), 150, out, D ** -0.5)
        torch.cuda.synchronize()
        ctx.check()
        at = 0
        for r, c in enumerate(chunk):
            kk = torch.from_numpy(PO.rotate(k[at: at + c].double().cpu().numpy(), total[r] + np.arange(c), 1e4)).to(torch.bfloat16)
            keys[r].append(kk.double().numpy())
            vals[r].append(v[at: at + c].double().cpu().numpy())
            total[r] += c
            K, V = np.concatenate(keys[r]), np.concatenate(vals[r])
            got_k = kc[r, : total[r]].double().cpu().numpy()
            assert (np.abs(got_k - K) <= 2.0 ** -7 * np.abs(K) + 1e-6).all() and (got_k != K).mean() < 1e-3
            K = got_k
            ref, _ = PO.attention(qr[at: at + c].double().cpu().numpy(), K, V, 0, 0, D ** -0.5)
            size, _ = PO.attention(qr[at: at + c].double().cpu().numpy(), K, np.abs(V), 0, 0, D ** -0.5)
            assert (np.abs(out[at: at + c].double().cpu().numpy() - ref) <= (2.0 ** -8 + 2.0 ** -12) * size + half_step(ref, "bf16")).all()
            at += c
        assert (out[n:] == 3).all()
    assert kv.tolist() == total and table.flatten().tolist() == list(range(2 * per))
    qt, kt, vt = (bf(rng.normal(size=(2, T, Hq, D))) for _ in range(3))
    kc.nan_to_num_()
    vc.nan_to_num_()
    att = torch.zeros_like(qt)
    cb.cascade_tree_attn(ctx, tree, qt, kc, vc, cap, kv, kt, vt, att, D ** -0.5)
    from oracle import cascade_oracle as O
    h = lambda t: t.float().cpu().numpy()  # noqa: E731
    ref = O.tree_attention(h(qt), h(kc), h(vc), np.array(total, np.int32), h(kt), h(vt), parent, D ** -0.5)
    assert np.abs(h(att) - ref).max() < 2e-2
    logits = torch.from_numpy(rng.normal(size=(2, 1024)).astype(np.float32)).to(G.DEV)
    tok, prob = i32([-9, -9]), torch.zeros(2, device=G.DEV)
    cb.cascade_sample(ctx, logits, torch.tensor([0.3, 0.8], device=G.DEV), tok, top_k=i32([50, 50]), prob=prob)
    ctx.check()
    for r, u in enumerate((0.3, 0.8)):
        t, p, _, gap = PO.sample(logits[r].cpu().numpy(), np.float32(u), 1.0, 50)
        assert int(tok[r]) == t and abs(float(prob[r]) - p) < 1e-6 * p and gap > 1e-9
    tree.close()
    ctx.close()


@pytest.mark.parametrize("window,sinks", [(0, 0), (70, 3)])
def test_more_blocks_than_multiprocessors(window, sinks):
    """32 key heads and requests of very different lengths: several hundred items, handed out one by one."""
    ctx = make_ctx("bf16", 32, 32, 64)
    c = Case("bf16", 32, 32, 64, 32, [17, 300, 1, 40, 0, 90, 33, 18, 20, 25], [400, 300, 700, 40, 9, 91, 64, 18, 500, 33], seed=5, pad=2)
    for _ in range(2):
        c.run(ctx, window, sinks)
        ctx.check()
        c.check(window, sinks)
        c.out.fill_(3.0)
        c.lse.fill_(3.0)
    ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("live", [{0: (20, 25)}, {40: (33, 70), 41: (1, 9), 95: (150, 150)}, {299: (40, 41)}, {}])
def test_padded_batch(dtype, live):
    """300 places, most of them without new tokens; one of those with a length out of bounds is reported all the same."""
    ctx = make_ctx(dtype, 4, 2, 64)
    q = [live.get(r, (0, 0))[0] for r in range(300)]
    kv = [live.get(r, (0, 3 * (r % 2)))[1] for r in range(300)]
    c = Case(dtype, 4, 2, 64, 8, q, kv, seed=3, pad=2)
    for _ in range(2):
        c.run(ctx, max_q=150, max_kv=200)
        ctx.check()
        c.check()
    c.kv[7 if 7 not in live else 8] = 10 ** 6
    c.run(ctx, max_q=150, max_kv=200)
    with pytest.raises(cb.CascadeError) as e:
        ctx.check()
    assert e.value.status == cb.ERR_BAD_PAGE
    c.check(requests=list(live))
    ctx.close()


def test_rows_summed_again_hold_nobody_past_the_wait_limit():
    """Every row meets a NaN and is computed again key by key, for much longer than the limit of the waits beside it."""
    H, D, page, n_req, q, kv = 40, 64, 16, 4, 20, 3000
    ctx = make_ctx("bf16", H, H, D)
    ctx.set_wait_limit(2_000_000)
    gen = torch.Generator(device=G.DEV)
    gen.manual_seed(1)
    pages = -(-kv // page)
    pool = torch.randn((2, n_req * pages, page, H, D), device=G.DEV, generator=gen).to(torch.bfloat16)
    pool[1, ::pages, 0] = float("nan")                       # the value of every request's first key
    cache = cb.PagedCache(pool[0], pool[1], torch.arange(n_req * pages, dtype=torch.int32, device=G.DEV).view(n_req, pages))
    x = torch.randn((n_req * q, H, D), device=G.DEV, generator=gen).to(torch.bfloat16)
    out, lse = torch.zeros_like(x), torch.zeros((n_req * q, H), device=G.DEV)
    begin, lens = i32(np.arange(n_req + 1) * q), i32([kv] * n_req)
    cb.cascade_paged_attn(ctx, cache, x, begin, lens, q, kv, out, 0.125, lse=lse)
    torch.cuda.synchronize()
    ctx.check()
    assert torch.isnan(out).all() and torch.isfinite(lse).all()
    pool[1, ::pages, 0] = 1.0
    cb.cascade_paged_attn(ctx, cache, x, begin, lens, q, kv, out, 0.125)
    torch.cuda.synchronize()
    ctx.check()
    assert torch.isfinite(out).all()
    ctx.close()


def test_two_contexts_at_once():
    """Chunks and single tokens of two contexts on two streams, the calls of each in order, results as when alone."""
    ctxs = [make_ctx("bf16", 16, 4, 128) for _ in range(2)]
    cases = [[Case("bf16", 16, 4, 128, 16, [33, 60, 17], [200, 333, 17], seed=1), Case("bf16", 16, 4, 128, 16, [1, 1], [300, 41], seed=2)],
             [Case("bf16", 16, 4, 128, 32, [130, 5], [130, 900], seed=3), Case("bf16", 16, 4, 128, 64, [2, 4], [77, 65], seed=4)]]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        for ctx, mine, st in zip(ctxs, cases, streams):
            with torch.cuda.stream(st):
                for c in mine:
                    cb.cascade_paged_attn(ctx, c.cache, c.q, c.q_begin, c.kv, max(c.q_len), max(c.kv_len), c.out, c.scale, lse=c.lse)
    torch.cuda.synchronize()
    for ctx, mine in zip(ctxs, cases):
        ctx.check()
        for c in mine:
            c.check()
        ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("q,kv", [([9, 4], [5, 0]), ([300], [290])])
def test_rows_before_the_first_key_and_the_widest_window(dtype, q, kv):
    """x - window + 1 of a row in front of the first key does not fit 32 bits."""
    ctx = make_ctx(dtype, 2, 2, 64)
    for window, sinks in ((2 ** 31 - 1, 0), (2 ** 31 - 1, 2 ** 31 - 1), (2 ** 31 - 2, 3), (4, 2 ** 31 - 1)):
        c = Case(dtype, 2, 2, 64, 16, q, kv, seed=len(q))
        c.run(ctx, window, sinks)
        ctx.check()
        c.check(window, sinks)
    ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_outputs_that_meet_the_queries_and_lengths_past_the_end_are_refused(dtype):
    L = cb.lib()
    ctx = make_ctx(dtype, 2, 2, 64)
    es = 2 if dtype == "bf16" else 4
    row, n = 128, 3                                       # rows of 128 elements, 400 elements apart
    buf = torch.zeros(8192, dtype=DT[dtype], device=G.DEV)
    idx = torch.zeros(64, dtype=torch.int32, device=G.DEV)
    p, i = buf.data_ptr(), idx.data_ptr()
    cache = cb.PagedCacheStruct(p + 6000 * es, p + 6000 * es, 8 * 128, 1, 8, i, 1)
    def call(at, mk=0, stride=400, q=1000):
        return L.cascade_paged_attn(ctx.handle, C.byref(cache), 1, n, p + q * es, stride, i, i, 1, mk, 0, 0, 1.0, p + at * es, None, None)
    for at in (1000, 1000 - n * row + 8, 1000 + 400 * 2 + row - 8, 1000 + row, 1000 + 400, 1000 + 400 + row):
        assert call(at) == cb.ERR_INVALID_ARG, at
    for at in (1000 - n * row, 1000 + 400 * 2 + row, 4000):
        assert call(at) == cb.OK, at
    assert call(1000 + row, stride=row + n * row) == cb.OK      # between two rows
    assert call(4000, mk=2 ** 31 - 65535) == cb.ERR_UNSUPPORTED_SHAPE
    assert call(4000, mk=2 ** 31 - 65536) == cb.OK
    ctx.check()
    ctx.close()


def test_refusals():
    L = cb.lib()
    ctx = make_ctx("bf16", 4, 2, 64)
    buf = torch.zeros(1 << 16, dtype=torch.int32, device=G.DEV)
    p = buf.data_ptr()
    def tables(n_req=1, n_tok=1, page=8, n_pages=4, width=2, slot=p, new=p, ctx_h=ctx.handle):
        return L.cascade_paged_tables(ctx_h, n_req, n_tok, page, n_pages, new, p, p, width, p, p, p, p, p, slot, p, None)
    for bad in (dict(n_req=0), dict(n_tok=-1), dict(page=0), dict(n_pages=0), dict(width=0), dict(slot=None), dict(new=None)):
        assert tables(**bad) == cb.ERR_INVALID_ARG, bad
    for bad in (dict(n_req=4097), dict(page=12), dict(n_pages=2 ** 28), dict(n_tok=2 ** 31 - 1)):
        assert tables(**bad) == cb.ERR_UNSUPPORTED_SHAPE, bad

    def cache(k=p, v=p, stride=1024, n_pages=4, page=8, table=p, width=2):
        return cb.PagedCacheStruct(k, v, stride, n_pages, page, table, width)

    bad_caches = [dict(k=None), dict(v=None), dict(k=p + 8), dict(stride=1023), dict(stride=1028), dict(n_pages=0), dict(page=0)]
    def append(n=1, q=None, qs=0, k=p, ks=128, v=p, vs=128, slot=p, pos=p, base=0.0, qo=None, qos=0, c=cache()):
        return L.cascade_paged_append(ctx.handle, C.byref(c), n, q, qs, k, ks, v, vs, slot, pos, base, qo, qos, None)
    for bad in [dict(n=0), dict(k=None), dict(v=p + 4), dict(ks=120), dict(vs=132), dict(slot=None), dict(pos=None), dict(base=0.5),
                dict(base=float("nan")), dict(base=float("inf")), dict(base=-3.0), dict(q=p, qs=256, qo=p, qos=256),
                dict(q=p, qs=256, base=1e4), dict(qo=p, qos=256, base=1e4), dict(q=p, qs=248, qo=p, qos=248, base=1e4),
                dict(q=p, qs=256, qo=p, qos=264, base=1e4)] + [dict(c=cache(**b)) for b in bad_caches]:
        assert append(**bad) == cb.ERR_INVALID_ARG, bad
    assert append(c=cache(page=12, stride=2048)) == cb.ERR_UNSUPPORTED_SHAPE

    def attn(n_req=1, n_tok=1, q=p, qs=256, qb=p, kv=p, mq=1, mk=1, w=0, s=0, scale=1.0, out=p, lse=None, c=cache()):
        return L.cascade_paged_attn(ctx.handle, C.byref(c), n_req, n_tok, q, qs, qb, kv, mq, mk, w, s, scale, out, lse, None)
    for bad in [dict(n_req=0), dict(n_tok=0), dict(q=None), dict(q=p + 2), dict(qs=255), dict(qs=260), dict(qb=None), dict(kv=None),
                dict(mq=0), dict(mk=-1), dict(w=-1), dict(s=-1), dict(scale=0.0), dict(scale=float("nan")), dict(scale=float("inf")),
                dict(out=None), dict(out=p + 8), dict(lse=p + 2), dict(c=cache(table=None)), dict(c=cache(width=0))] + \
               [dict(c=cache(**b)) for b in bad_caches]:
        assert attn(**bad) == cb.ERR_INVALID_ARG, bad
    assert attn(n_req=4097) == cb.ERR_UNSUPPORTED_SHAPE
    torch.cuda.synchronize()
    assert int(buf.abs().sum()) == 0
    ctx.check()
    ctx.close()
