"""GPU parity of the paged attention's gradient against the formula in 64 bits, within bounds that count its roundings."""
import math

import numpy as np
import pytest
import torch

from oracle import train_oracle as TO
from paper_2605_07230_b200 import binding as cb
from tests import gpu_util as G

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def i32(x):
    return torch.as_tensor(np.asarray(x, np.int32), device=G.DEV)


class Call:
    """One pass: requests of q_len new tokens over kv_len keys in a pool of scattered pages; stacked queries and gradients."""

    def __init__(self, q_len, kv_len, Hq=2, Hkv=2, D=64, dtype="bf16", page=16, window=0, sinks=0, seed=0, pad=0, own_rows=True, gap=0,
                 scale=None, size=1.0):
        rng = np.random.default_rng(seed)
        gen = torch.Generator(device=G.DEV).manual_seed(seed)
        normal = lambda *s: (size * torch.randn(s, device=G.DEV, generator=gen)).to(DT[dtype])   # noqa: E731
        self.q_len, self.kv_len_host, self.window, self.sinks, self.dtype, self.page = list(q_len), list(kv_len), window, sinks, dtype, page
        self.Hq, self.Hkv, self.D, self.scale = Hq, Hkv, D, D ** -0.5 if scale is None else scale
        counts = [-(-n // page) for n in kv_len]
        n_pages = sum(counts) + 2
        ids = rng.permutation(n_pages)
        self.table_host = np.full((len(q_len), max(counts + [1])), -1, np.int32)
        at = 0
        for r, c in enumerate(counts):
            self.table_host[r, :c] = ids[at: at + c]
            at += c
        n = max(1, sum(q_len) + pad)
        nan = lambda *s: torch.full(s, float("nan"), device=G.DEV, dtype=DT[dtype])              # noqa: E731
        self.qkv = normal(n, (Hq + 2 * Hkv) * D + gap)
        self.q = self.qkv[:, : Hq * D].view(n, Hq, D)
        self.k_pages, self.v_pages = normal(n_pages, page, Hkv, D), normal(n_pages, page, Hkv, D)
        self.table, self.q_begin = i32(self.table_host), i32(np.concatenate([[0], np.cumsum(q_len)]))
        self.kv_len = i32(kv_len)
        first = np.cumsum([0] + [k + (3 if own_rows else 0) for k in kv_len])       # (rows between the requests belong to nobody)
        self.first = first[:-1]
        self.k_begin = i32(self.first) if own_rows else None
        self.out, self.d_out = nan(n, Hq, D), normal(n, Hq, D)
        self.lse = torch.full((n, Hq), float("nan"), device=G.DEV)
        self.scratch = torch.full((n, Hq, 2), float("nan"), device=G.DEV)
        n_kv = max(int(first[-1]), 1)
        if own_rows:
            self.dq, self.dk, self.dv = nan(n, Hq, D), nan(n_kv, Hkv, D), nan(n_kv, Hkv, D)
        else:                                                                       # parts of one stacked gradient
            self.d_qkv = nan(max(n, n_kv), (Hq + 2 * Hkv) * D + gap)
            part = lambda a, h, m: self.d_qkv[:m, a: a + h * D].view(m, h, D)                    # noqa: E731
            self.dq, self.dk, self.dv = part(0, Hq, n), part(Hq * D, Hkv, n_kv), part((Hq + Hkv) * D, Hkv, n_kv)
        self.max_q, self.max_kv = max(list(q_len) + [1]), max(kv_len)
        self.ctx = cb.Context(cb.BF16 if dtype == "bf16" else cb.F32, 1, 1, 64, 64, Hq, Hkv, D, 64)
        self.cache = cb.PagedCache(self.k_pages, self.v_pages, self.table)

    def forward(self):
        cb.cascade_paged_attn(self.ctx, self.cache, self.q, self.q_begin, self.kv_len, self.max_q, self.max_kv, self.out, self.scale,
                              window=self.window, sinks=self.sinks, lse=self.lse)

    def backward(self):
        cb.cascade_paged_attn_grad(self.ctx, self.cache, self.q, self.q_begin, self.kv_len, self.max_q, self.max_kv, self.out, self.lse,
                                   self.d_out, self.scratch, self.dq, self.dk, self.dv, self.scale, window=self.window, sinks=self.sinks,
                                   k_begin=self.k_begin)

    def run(self):
        self.forward()
        self.backward()
        self.ctx.check()
        return self

    def request(self, r):
        """Rows, keys and values of request r in 64 bits."""
        a, n, L = int(self.q_begin[r]), self.q_len[r], self.kv_len_host[r]
        j = torch.arange(L, device=G.DEV)
        page = torch.as_tensor(self.table_host[r].astype(np.int64), device=G.DEV)[j // self.page]
        rows = [t[a: a + n].double() for t in (self.q, self.d_out, self.out, self.lse)]
        return rows, self.k_pages[page, j % self.page].double(), self.v_pages[page, j % self.page].double()

    def sees(self, r, there=None):
        n, L = self.q_len[r], self.kv_len_host[r]
        x, j = (L - n + torch.arange(n, device=G.DEV))[:, None], torch.arange(L, device=G.DEV)[None, :]
        ok = j <= x
        if self.window:
            ok = ok & ((j > x - self.window) | (j < self.sinks))
        return ok if there is None else ok & there[None, :]

    def exact(self, r, there=None):
        """dq, dk, dv of request r, and the sums of their terms' sizes."""
        (q, g, o, lse), k, v = self.request(r)
        see, rep = self.sees(r, there), self.Hq // self.Hkv
        k, v = (t.repeat_interleave(rep, 1) for t in (k, v))
        s = torch.einsum("ihd,jhd->hij", q, k) * self.scale
        p = torch.where(see, torch.exp(s - lse.T[:, :, None]), 0.0)
        dp, delta = torch.einsum("ihd,jhd->hij", g, v), (g * o).sum(-1).T[:, :, None]
        ds = torch.where(see, p * (dp - delta), 0.0) * self.scale
        big = p * (torch.einsum("ihd,jhd->hij", g.abs(), v.abs()) + (g.abs() * o.abs()).sum(-1).T[:, :, None]) * self.scale
        fold = lambda t: t.view(t.shape[0], self.Hkv, rep, self.D).sum(2)                        # noqa: E731
        res = [torch.einsum("hij,jhd->ihd", ds, k), fold(torch.einsum("hij,ihd->jhd", ds, q)), fold(torch.einsum("hij,ihd->jhd", p, g))]
        size = [torch.einsum("hij,jhd->ihd", big, k.abs()), fold(torch.einsum("hij,ihd->jhd", big, q.abs())),
                fold(torch.einsum("hij,ihd->jhd", p, g.abs()))]
        return res, size

    def got(self, r):
        a, n, f, L = int(self.q_begin[r]), self.q_len[r], int(self.first[r]), self.kv_len_host[r]
        return [self.dq[a: a + n].double(), self.dk[f: f + L].double(), self.dv[f: f + L].double()]

    def tolerance(self, r, size, want):
        """A score is off by its D roundings of terms that sum to at most S (in 32 bits, a tensor core's additions counted twice),
        its exponential by that, by its argument's three roundings and by 2^-22 of its own; the weight's gradient by D roundings of
        its parts; both go to the operands' type for a product (half a step, and a hundredth of one for an exponential that is off by
        3e-6), and n terms are added.  One rounding of the result."""
        (q, g, o, lse), k, v = self.request(r)
        if not len(q) or not len(k):
            return [torch.zeros_like(w) for w in want]
        half = 2.0**-8 if self.dtype == "bf16" else 2.0**-24
        S = float(q.abs().amax((0, 1)) @ k.abs().amax((0, 1))) * self.scale
        arg = S + float(lse[lse.isfinite()].abs().max()) if bool(lse.isfinite().any()) else S
        n = max(len(q) * (self.Hq // self.Hkv), len(k))
        e = 2 * self.D * 2.0**-24 * S + 3 * arg * 2.0**-24 + 2.0**-22 + 2 * (self.D + n) * 2.0**-24
        return [s * (half * 1.01 + e) * (1 + half) + half * w.abs() + 1e-30 for s, w in zip(size, want)]

    def check(self, there=None):
        for r in range(len(self.q_len)):
            want, size = self.exact(r, there)
            for name, x, w, t in zip(("dq", "dk", "dv"), self.got(r), want, self.tolerance(r, size, want)):
                bad = ~((x - w).abs() <= t)
                assert not bad.any(), (r, name, bad.nonzero()[:3].tolist(), x[bad][:3].tolist(), w[bad][:3].tolist(), t[bad][:3].tolist())
        n = sum(self.q_len)
        assert self.dq[n:].isnan().all()                                            # rows behind the last sequence stay as they were
        if self.k_begin is not None:
            rest = torch.ones(self.dk.shape[0], dtype=torch.bool, device=G.DEV)
            for f, L in zip(self.first, self.kv_len_host):
                rest[int(f): int(f) + L] = False
            assert self.dk[rest].isnan().all() and self.dv[rest].isnan().all()


def test_the_reference_is_the_checker_s():
    c = Call([5, 3], [9, 2], Hq=4, Hkv=2, dtype="f32", window=4, sinks=2).run()
    for r in range(2):
        (q, g, o, lse), k, v = c.request(r)
        a, b = TO.attention_grad(*(t.cpu().numpy() for t in (q, k, v, g)), 4, 2, c.scale, out=o.cpu().numpy(), lse=lse.cpu().numpy())
        want, size = c.exact(r)
        for x, y in zip(list(a) + list(b), want + size):
            assert np.allclose(x, y.cpu().numpy(), atol=1e-12)


HEADS = [(2, 2, 64), (2, 2, 128), (8, 2, 128), (5, 1, 64), (6, 2, 128)]
LENGTHS = [([1], [1]), ([64], [64]), ([127, 1, 130], [127, 1, 130]), ([3, 70, 1], [200, 70, 129]), ([300], [300]), ([129], [513]),
           ([7, 0, 5], [40, 30, 2]), ([1, 2, 1], [260, 0, 1])]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,D", HEADS)
@pytest.mark.parametrize("q_len,kv_len", LENGTHS)
def test_gradients(q_len, kv_len, Hq, Hkv, D, dtype):
    Call(q_len, kv_len, Hq, Hkv, D, dtype, seed=len(q_len) + sum(kv_len), pad=2).run().check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window,sinks", [(1, 0), (16, 0), (100, 3), (128, 128), (200, 150), (1000, 4), (37, 129)])
@pytest.mark.parametrize("Hq,Hkv,D", [(2, 2, 128), (8, 2, 64)])
def test_windows_and_first_tokens(window, sinks, Hq, Hkv, D, dtype):
    Call([300, 65, 10], [300, 500, 700], Hq, Hkv, D, dtype, window=window, sinks=sinks, seed=window, pad=1).run().check()


@pytest.mark.parametrize("page", [8, 24, 48, 64, 128, 256])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_page_sizes(page, dtype):
    Call([140, 33], [270, 33], 4, 2, 128, dtype, page=page, seed=page).run().check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("gap", [0, 8])
def test_whole_sequences_into_one_stacked_gradient(dtype, gap):
    c = Call([100, 3, 257], [100, 3, 257], 4, 2, 64, dtype, own_rows=False, gap=gap, seed=3)
    c.run().check()
    assert c.d_qkv[:, (c.Hq + 2 * c.Hkv) * c.D:].isnan().all()


def test_many_query_heads_a_key_head():
    Call([9, 40], [30, 40], 128, 1, 64, seed=5).run().check()
    Call([9, 40], [30, 40], 96, 2, 128, seed=6).run().check()
    Call([17], [33], 100, 1, 128, seed=7).run().check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_requests_some_without_tokens(dtype):
    rng = np.random.default_rng(1)
    q = rng.integers(0, 40, 90)
    q[rng.random(90) < 0.4] = 0
    kv = q + rng.integers(0, 60, 90)
    kv[:3] = 0
    Call(q.tolist(), kv.tolist(), 2, 1, 64, dtype, seed=2, pad=5).run().check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("q_len,kv_len", [([4], [0]), ([3, 0, 0], [0, 0, 7]), ([0, 0], [0, 5])])
def test_requests_without_keys_or_rows(q_len, kv_len, dtype):
    Call(q_len, kv_len, 2, 1, 64, dtype, pad=1).run().check()


def test_more_items_than_a_launch_holds_at_once():
    """Several items a block, and blocks that go on with the other pass; the same bits every time."""
    rng = np.random.default_rng(3)
    q = rng.integers(1, 280, 30).tolist()
    c = Call(q, [n + int(rng.integers(0, 60)) for n in q], 20, 20, 64, seed=16).run()
    c.check()
    first = [t.clone() for r in range(30) for t in c.got(r)]
    for _ in range(3):
        c.backward()
    c.ctx.check()
    assert all(torch.equal(a, b) for a, b in zip(first, [t for r in range(30) for t in c.got(r)]))


def test_long_sums_key_by_key_beside_short_waits():
    """A value that is no number has most keys of a long sequence summed again: no wait gives up meanwhile."""
    c = Call([1500], [1500], 4, 2, 128, seed=17)
    c.forward()
    c.d_out[1400, 0, 3] = float("nan")
    c.ctx.set_wait_limit(3_000_000)
    c.backward()
    c.ctx.check()
    got = c.got(0)
    assert got[2][:1401, 0].isnan().any(-1).all() and got[2][1401:].isfinite().all() and got[2][:, 1].isfinite().all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_bounds_far_above_the_lengths_change_nothing(dtype):
    c = Call([70, 1, 0, 133], [70, 40, 9, 300], 4, 2, 64, dtype, seed=18).run()
    first = [t.clone() for r in range(4) for t in c.got(r)]
    c.max_q, c.max_kv = 1 << 20, c.table.shape[1] * 16 * 1000
    c.backward()
    c.ctx.check()
    assert all(torch.equal(a, b) for a, b in zip(first, [t for r in range(4) for t in c.got(r)]))


@pytest.mark.parametrize("D", [64, 128])
def test_fp32_numbers_of_all_sizes(D):
    """Values and output gradients of 2^-40 to 2^40: every element keeps its own 24 bits."""
    c = Call([150], [190], 2, 1, D, "f32", seed=19)
    rng = np.random.default_rng(20)
    power = lambda t: t.mul_(torch.as_tensor(2.0 ** rng.integers(-40, 41, tuple(t.shape)).astype(np.float32), device=G.DEV))   # noqa: E731
    power(c.v_pages)
    power(c.d_out)
    c.run().check()


@pytest.mark.parametrize("window,sinks", [(0, 0), (300, 5)])
@pytest.mark.parametrize("q_len,kv_len,Hq,Hkv,D", [([1000], [1000], 1, 1, 64), ([500, 31], [500, 700], 8, 1, 128), ([900], [900], 10, 2, 64),
                                                   ([330, 330], [400, 330], 2, 2, 128), ([3], [2000], 1, 1, 64), ([700], [40], 4, 1, 64),
                                                   ([2000], [2000], 8, 1, 64), ([300, 0, 260], [310, 0, 290], 32, 1, 128)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_few_tiles_with_long_walks(q_len, kv_len, Hq, Hkv, D, window, sinks, dtype):
    """A tile's steps are shared out over a cluster: the sums, and the same bits every time."""
    c = Call(q_len, kv_len, Hq, Hkv, D, dtype, window=window, sinks=sinks, seed=24).run()
    c.check()
    first = [t.clone() for r in range(len(q_len)) for t in c.got(r)]
    for _ in range(3):
        c.backward()
    c.ctx.check()
    assert all(torch.equal(a, b) for a, b in zip(first, [t for r in range(len(q_len)) for t in c.got(r)]))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_value_that_is_no_number_in_a_long_walk(dtype):
    c = Call([1000], [1000], 8, 1, 64, dtype, seed=25)
    c.forward()
    c.d_out[900, 0, 7] = float("nan")
    c.backward()
    c.ctx.check()
    dq, dk, dv = c.got(0)
    assert dq[900, 0].isnan().any() and dq[:900].isfinite().all() and dq[901:].isfinite().all() and dq[:, 1].isfinite().all()
    assert dv[:901, 0, 7].isnan().all() and dv[901:].isfinite().all() and dk[901:].isfinite().all()


def test_calls_of_both_types_side_by_side():
    calls = [Call([400], [400], 8, 8, 128, "bf16", seed=21), Call([300], [300], 4, 4, 64, "f32", seed=22), Call([200, 90], [200, 90], 4, 4, 128, "f32", seed=23)]
    for c in calls:
        c.forward()
    streams = [torch.cuda.Stream() for _ in calls]
    torch.cuda.synchronize()
    for _ in range(4):
        for c, s in zip(calls, streams):
            with torch.cuda.stream(s):
                c.backward()
    torch.cuda.synchronize()
    for c in calls:
        c.ctx.check()
        c.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_steep_scores(dtype):
    """Weights near 0 and 1 (scores of a size of a hundred)."""
    Call([200], [200], 2, 1, 128, dtype, size=3.5, seed=11).run().check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
def test_what_a_row_does_not_see_does_not_reach_it(dtype, D):
    """NaN and infinities in keys, values, queries and output gradients that nobody sees."""
    clean = Call([150, 40], [150, 200], 2, 1, D, dtype, window=50, sinks=2, seed=4, pad=3).run()
    c = Call([150, 40], [150, 200], 2, 1, D, dtype, window=50, sinks=2, seed=4, pad=3)
    for t in (c.k_pages, c.v_pages):
        for r, L in enumerate(c.kv_len_host):                       # rows of the last page behind the last key, and free pages
            last = int(c.table_host[r, (L - 1) // 16])
            if L % 16:
                t[last, L % 16:] = float("nan")
        used = set(c.table_host[c.table_host >= 0].tolist())
        for p in range(t.shape[0]):
            if p not in used:
                t[p] = float("inf")
        t[int(c.table_host[1, 20 // 16]), 20 % 16] = float("nan")   # key 20 of the second request: outside every row's window
    c.q[190:] = float("nan")                                        # rows behind the last sequence
    c.d_out[190:] = float("inf")
    c.run()
    # the sums beside such values are taken key by key, in another order: held to the bounds of the formula at the clean values
    for mine, theirs in ((c.q, clean.q), (c.d_out, clean.d_out), (c.k_pages, clean.k_pages), (c.v_pages, clean.v_pages)):
        mine.copy_(theirs)
    c.check()
    assert not c.dk[173].any() and not c.dv[173].any()              # nobody sees it


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("where", ["key", "value", "query", "d_out"])
def test_a_value_that_is_no_number_stays_with_those_that_see_it(where, dtype):
    clean = Call([150], [150], 4, 2, 64, dtype, seed=8).run()
    c = Call([150], [150], 4, 2, 64, dtype, seed=8)
    bad = 70
    pool = {"key": c.k_pages, "value": c.v_pages}.get(where)
    if pool is not None:
        pool[int(c.table_host[0, bad // 16]), bad % 16, 0, 5] = float("nan")         # key 70 of key head 0
        c.forward()
    else:
        c.forward()
        (c.q if where == "query" else c.d_out)[bad, 1, 5] = float("nan")             # row 70 of query head 1, read by key head 0
    c.backward()
    c.ctx.check()
    same = lambda a, b, t: ((a - b).abs() <= t).all()                                # noqa: E731
    for mine, theirs in ((c.q, clean.q), (c.d_out, clean.d_out), (c.k_pages, clean.k_pages), (c.v_pages, clean.v_pages)):
        mine.copy_(theirs)                                                           # the formula at the clean values
    want, size = c.exact(0)
    tol = c.tolerance(0, size, want)
    got = c.got(0)
    # key head 1 and its query heads do not meet it
    assert torch.equal(c.dq[:, 2:], clean.dq[:, 2:]) and torch.equal(c.dk[:150, 1], clean.dk[:150, 1]) and torch.equal(c.dv[:150, 1], clean.dv[:150, 1])
    if pool is not None:
        assert same(got[0][:bad], want[0][:bad], tol[0][:bad])                       # rows in front of it
        assert got[0][bad:, :2].isnan().any(-1).all()                                # rows that see it
        assert got[1][bad, 0].isnan().any()
    else:
        assert same(got[1][bad + 1:], want[1][bad + 1:], tol[1][bad + 1:]) and same(got[2][bad + 1:], want[2][bad + 1:], tol[2][bad + 1:])
        assert got[1][: bad + 1, 0].isnan().any(-1).all()                            # keys that it sees
        others = torch.arange(150, device=G.DEV) != bad
        assert same(got[0][others], want[0][others], tol[0][others]) and same(got[0][bad, [0, 2, 3]], want[0][bad, [0, 2, 3]], tol[0][bad, [0, 2, 3]])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_pages_outside_the_pool(dtype):
    for bad_page in (-1, 2**31 - 1, -2**31):
        c = Call([60, 30], [60, 90], 2, 1, 128, dtype, seed=9)
        there = [torch.ones(n, dtype=torch.bool, device=G.DEV) for n in c.kv_len_host]
        c.table[1, 2] = bad_page                                    # keys 32 .. 47 of the second request
        c.forward()
        with pytest.raises(cb.CascadeError):
            c.ctx.check()
        c.backward()
        with pytest.raises(cb.CascadeError) as e:
            c.ctx.check()
        assert e.value.status == cb.ERR_BAD_PAGE
        there[1][32:48] = False
        for r in range(2):
            want, size = c.exact(r, there[r])
            for x, w, t in zip(c.got(r), want, c.tolerance(r, size, want)):
                assert ((x - w).abs() <= t).all()
        assert not c.got(1)[1][32:48].any() and not c.got(1)[2][32:48].any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_requests_outside_what_was_given_are_left_out(dtype):
    def spoiled(change):
        c = Call([20, 30, 10], [20, 50, 10], 2, 1, 64, dtype, seed=10)
        c.forward()
        c.ctx.check()
        change(c)
        c.backward()
        with pytest.raises(cb.CascadeError) as e:
            c.ctx.check()
        assert e.value.status == cb.ERR_BAD_PAGE
        for r in (0, 2):
            want, size = c.exact(r)
            for x, w, t in zip(c.got(r), want, c.tolerance(r, size, want)):
                assert ((x - w).abs() <= t).all()
        assert all(x[:30].isnan().all() for x in c.got(1))              # (without k_begin the next request's rows follow)

    def assign(name, value):
        def change(c):
            getattr(c, name)[1] = value
        return change

    spoiled(assign("k_begin", -1))
    spoiled(assign("k_begin", 2**31 - 1))
    spoiled(assign("kv_len", 10**6))
    spoiled(assign("kv_len", -3))

    def bound(c):
        c.max_kv = 49
    spoiled(bound)

    def rows_of_the_pass(c):                                        # keys that are not all of this pass, without rows of their own
        c.k_begin = None
        c.first = np.array([0, 20, 50])
    spoiled(rows_of_the_pass)


@pytest.mark.parametrize("q_len,H,D,dtype", [([90, 200], 4, 128, "f32"), ([1000], 1, 64, "f32"), ([90, 200], 4, 64, "bf16")])
def test_a_context_whose_first_call_is_recorded(q_len, H, D, dtype):
    c = Call(q_len, q_len, H, H, D, dtype, seed=26)
    c.forward()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.backward()
    graph.replay()
    torch.cuda.synchronize()
    c.ctx.check()
    c.check()
    first = [t.clone() for r in range(len(q_len)) for t in c.got(r)]
    c.backward()
    assert all(torch.equal(a, b) for a, b in zip(first, [t for r in range(len(q_len)) for t in c.got(r)]))


def test_recorded_and_replayed_on_another_stream():
    c = Call([90, 200], [90, 200], 4, 4, 128, seed=12)
    c.forward()
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    c.backward()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        c.backward()
    first = [t.clone() for r in range(2) for t in c.got(r)]
    for t in (c.dq, c.dk, c.dv):
        t.fill_(float("nan"))
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    c.ctx.check()
    assert all(torch.equal(a, b) for a, b in zip(first, c.got(0) + c.got(1)))        # and the same bits every time
    c.d_out.copy_(c.d_out.flip(0))
    graph.replay()
    torch.cuda.synchronize()
    c.check()


def test_two_contexts_on_two_streams():
    calls = [Call([300, 50], [300, 80], 4, 2, 128, seed=s) for s in (13, 14)]
    streams = [torch.cuda.Stream() for _ in calls]
    torch.cuda.synchronize()
    for _ in range(3):
        for c, s in zip(calls, streams):
            with torch.cuda.stream(s):
                c.forward()
                c.backward()
    torch.cuda.synchronize()
    for c in calls:
        c.ctx.check()
        c.check()


def test_gradient_by_differences():
    """The gradient is that of the forward call itself."""
    c = Call([50, 20], [50, 60], 4, 2, 64, "f32", window=30, sinks=2, seed=15).run()
    gen = torch.Generator(device=G.DEV).manual_seed(1)
    dq, dk, dv = c.dq.clone(), [x.clone() for x in (c.got(0)[1], c.got(1)[1])], [x.clone() for x in (c.got(0)[2], c.got(1)[2])]
    ways = [torch.randn(t.shape, device=G.DEV, generator=gen) for t in (c.q, c.k_pages, c.v_pages)]
    want = (dq[:70].double() * ways[0][:70].double()).sum()
    for r in range(2):
        j = torch.arange(c.kv_len_host[r], device=G.DEV)
        page = torch.as_tensor(c.table_host[r].astype(np.int64), device=G.DEV)[j // 16]
        want = want + (dk[r] * ways[1][page, j % 16].double()).sum() + (dv[r] * ways[2][page, j % 16].double()).sum()
    f, e = [], 1e-2
    base = [t.clone() for t in (c.q, c.k_pages, c.v_pages)]
    for s in (1, -1, 2, -2):
        for t, b, w in zip((c.q, c.k_pages, c.v_pages), base, ways):
            t.copy_(b + s * e * w)
        c.forward()
        f.append((c.out[:70].double() * c.d_out[:70].double()).sum())
    slope = (8 * (f[0] - f[1]) - (f[2] - f[3])) / (12 * e)          # fourth order: the error is that of the outputs' roundings
    noise = 9 * float((c.out[:70].double().abs() * c.d_out[:70].double().abs()).sum()) * 2.0**-20 / (6 * e)
    assert abs(float(slope - want)) <= noise + 1e-3 * abs(float(want))


def test_binding_checks_what_it_is_given():
    c = Call([20], [20])
    c.forward()
    for name, bad in (("out", c.out[:, :1]), ("lse", c.lse.double()), ("d_out", c.d_out.float()), ("scratch", c.scratch[..., 0]),
                      ("dq", c.dq.float()), ("dk", c.dk[:, :, :32]), ("k_begin", c.k_begin.long()), ("dv", c.dv.cpu())):
        keep = getattr(c, name)
        setattr(c, name, bad)
        with pytest.raises(ValueError):
            c.backward()
        setattr(c, name, keep)
    c.dv = c.dk
    with pytest.raises(cb.CascadeError):
        c.backward()
