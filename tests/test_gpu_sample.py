"""GPU parity of cascade_sample against its 64-bit restatement.  Tokens and kept counts are exact; a row whose uniform (or a
threshold) falls within 1e-9 of a boundary is not a test of anything and does not occur with these seeds."""

import numpy as np
import pytest
import torch

from oracle import paged_oracle as PO
from paper_2605_07230_b200 import binding as cb
from tests import gpu_util as G

pytestmark = pytest.mark.gpu


def make_ctx(V):
    return cb.Context(cb.F32, 1, 1, 64, 64, 1, 1, 64, V)


def dev(x, dt):
    return None if x is None else torch.as_tensor(np.asarray(x), device=G.DEV).to(dt).contiguous()


def run(ctx, logits, u, T=None, k=None, p=None, mp=None, stream=None):
    n = logits.shape[0]
    tok = torch.full((n,), -9, dtype=torch.int32, device=G.DEV)
    prob = torch.full((n,), -9.0, device=G.DEV)
    kept = torch.full((n,), -9, dtype=torch.int32, device=G.DEV)
    f, i = torch.float32, torch.int32
    cb.cascade_sample(ctx, logits, dev(u, f), tok, dev(T, f), dev(k, i), dev(p, f), dev(mp, f), prob, kept)
    torch.cuda.synchronize()
    ctx.check()
    return tok.cpu().numpy(), prob.cpu().numpy(), kept.cpu().numpy()


def compare(logits, got, u, T=None, k=None, p=None, mp=None, gap_min=1e-9):
    rows = logits.double().cpu().numpy()
    at = lambda x, r, off: off if x is None else np.float64(np.asarray(x)[r])  # noqa: E731
    for r in range(rows.shape[0]):
        t, pr, n, gap = PO.sample(rows[r], at(u, r, 0.0), at(T, r, 1.0), int(at(k, r, 0)), at(p, r, 1.0), at(mp, r, 0.0))
        assert gap > gap_min or n <= 1 or u[r] == 0, (r, gap)
        assert (got[0][r], got[2][r]) == (t, n), (r, got[0][r], t, got[2][r], n, gap)
        assert abs(got[1][r] - pr) <= 2.0 ** -23 * pr + 1e-12, (r, got[1][r], pr)


def cluster_logits(rng, n, V, noise=0.3):
    level = rng.normal(0, 2.6, (n, 256))
    return (level[:, np.arange(V) % 256] + rng.normal(0, noise, (n, V))).astype(np.float32)


SETTINGS = [dict(), dict(T=0.7), dict(k=1), dict(k=50), dict(p=0.9), dict(p=0.05, T=1.5), dict(mp=0.05), dict(k=200, p=0.8, mp=0.01, T=1.2),
            dict(k=7, p=0.5)]


@pytest.mark.parametrize("V,n", [(8, 9), (128, 5), (1000, 7), (1024, 3), (16384, 6), (49152, 2), (65536, 4), (131080, 2)])
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
def test_settings(V, n, dt):
    rng = np.random.default_rng(V)
    ctx = make_ctx(V)
    logits = torch.from_numpy(cluster_logits(rng, n, V)).to(G.DEV).to(dt)
    for s in SETTINGS:
        u = rng.random(n).astype(np.float32)
        kw = {name: np.full(n, x, np.int32 if name == "k" else np.float32) for name, x in s.items()}
        compare(logits, run(ctx, logits, u, **kw), u, **kw)
    ctx.close()


def test_settings_per_row_and_rows_apart():
    V, n = 2048 + 40, 40
    rng = np.random.default_rng(3)
    ctx = make_ctx(V)
    wide = torch.from_numpy(cluster_logits(rng, n, V + 7)).to(G.DEV)
    logits = wide[:, 3:3 + V]                                # 4 bytes off alignment, rows 7 elements further apart
    u = rng.random(n).astype(np.float32)
    kw = dict(T=rng.choice([0.0, -1.0, 0.3, 1.0, 2.0], n).astype(np.float32), k=rng.choice([-3, 0, 1, 5, 400, V, V + 9], n).astype(np.int32),
              p=rng.choice([0.3, 0.95, 1.0, 7.0], n).astype(np.float32), mp=rng.choice([-1.0, 0.0, 0.02, 0.4], n).astype(np.float32))
    before = wide.clone()
    compare(logits, run(ctx, logits, u, **kw), u, **kw)
    assert torch.equal(wide, before)
    ctx.close()


@pytest.mark.parametrize("V", [4096, 16384, 65536])
@pytest.mark.parametrize("T", [0.02, 1.0, 30.0])
def test_nucleus_in_a_crowd(V, T):
    """One logit far above thousands that nearly agree: the threshold's step, and the estimate's band, hold too many tokens."""
    rng = np.random.default_rng(V)
    ctx = make_ctx(V)
    x = (1e-3 * rng.normal(size=(4, V))).astype(np.float32)
    x[np.arange(4), rng.integers(0, V, 4)] = 30.0
    x[2] = np.round(x[2] * 256) / 256                        # and ties
    logits = torch.from_numpy(x).to(G.DEV)
    u = rng.random(4).astype(np.float32)
    for p in (0.3, 0.7):
        kw = dict(T=np.full(4, T, np.float32), p=np.full(4, p, np.float32))
        compare(logits, run(ctx, logits, u, **kw), u, **kw)
        kw["k"] = np.full(4, 5000, np.int32)
        compare(logits, run(ctx, logits, u, **kw), u, **kw)
    ctx.close()


@pytest.mark.parametrize("n", [149, 600, 4096, 4100])
def test_many_rows_with_settings_of_their_own(n):
    V = 96
    rng = np.random.default_rng(n)
    ctx = make_ctx(V)
    logits = torch.from_numpy(cluster_logits(rng, n, V)).to(G.DEV)
    u = rng.random(n).astype(np.float32)
    kw = dict(T=rng.choice([0.0, 0.7, 1.0, 1.4], n).astype(np.float32), k=rng.choice([0, 1, 7, V], n).astype(np.int32),
              p=rng.choice([0.5, 0.9, 1.0], n).astype(np.float32), mp=rng.choice([0.0, 0.05], n).astype(np.float32))
    compare(logits, run(ctx, logits, u, **kw), u, **kw)
    compare(logits, run(ctx, logits, u, p=kw["p"]), u, p=kw["p"])
    compare(logits, run(ctx, logits, u, T=np.zeros(n, np.float32)), u, T=np.zeros(n, np.float32))
    ctx.close()


def test_every_token_gets_its_share():
    """Uniforms on a fine grid over one row: the counts are the kept probabilities."""
    V, n = 64, 4096
    rng = np.random.default_rng(11)
    ctx = make_ctx(V)
    row = rng.normal(0, 1.5, V).astype(np.float32)
    logits = torch.from_numpy(row).to(G.DEV).expand(n, V).contiguous()
    u = ((np.arange(n) + 0.5) / n).astype(np.float32)
    tok, prob, kept = run(ctx, logits, u, k=np.full(n, 20, np.int32))
    p = np.exp(row.astype(np.float64))
    p[row < np.sort(row)[V - 20]] = 0
    p /= p.sum()
    assert np.abs(np.bincount(tok, minlength=V) / n - p).max() <= 1.0 / n and (kept == 20).all()
    assert (np.diff(tok) >= 0).all()                         # the inverse of a cumulative sum in index order
    assert np.abs(prob - p[tok]).max() < 1e-6
    ctx.close()


def test_ties_and_rows_without_a_choice():
    V = 512
    inf, nan = np.inf, np.nan
    rng = np.random.default_rng(5)
    rows = np.zeros((12, V), np.float32)
    rows[1] = np.round(rng.normal(0, 2, V))                  # many equal logits
    rows[2, ::2] = -0.0                                      # zeros of both signs are one value
    rows[3] = -inf
    rows[4] = nan
    rows[5] = -inf
    rows[5, 77] = -3e38
    rows[6] = nan
    rows[6, [5, 9]] = 1.0
    rows[7, [3, 400]] = inf
    rows[8] = np.finfo(np.float32).min                       # a mask of the type's lowest value ...
    rows[8, 10:20] = rng.normal(size=10)                     # ... around a few real ones
    rows[9] = np.finfo(np.float32).min
    rows[10] = rng.normal(0, 1e-30, V)
    rows[11] = np.linspace(-3e38, 3e38, V)
    ctx = make_ctx(V)
    logits = torch.from_numpy(rows).to(G.DEV)
    n = len(rows)
    u = np.array([0.503, 0.21, 0.77, 0.5, 0.5, 0.5, 0.7, 0.6, 0.4, 0.123, 0.9, 0.3], np.float32)
    for kw in (dict(), dict(k=np.full(n, 3, np.int32)), dict(p=np.full(n, 0.3, np.float32)), dict(mp=np.full(n, 0.5, np.float32)),
               dict(k=np.full(n, 3, np.int32), p=np.full(n, 0.3, np.float32), mp=np.full(n, 1.0, np.float32)),
               dict(T=np.zeros(n, np.float32))):
        compare(logits, run(ctx, logits, u, **kw), u, **kw)
    tok, prob, kept = run(ctx, logits, u)
    assert (tok[3], prob[3], kept[3]) == (-1, 0.0, 0) and (tok[4], kept[4]) == (-1, 0)
    assert tok[7] == 400 and prob[7] == 0.5
    ctx.close()


def test_odd_settings():
    """Uniforms outside [0,1), settings that are NaN or out of range, the smallest and largest temperatures."""
    V = 256
    rng = np.random.default_rng(8)
    ctx = make_ctx(V)
    row = rng.normal(0, 2, V).astype(np.float32)
    logits = torch.from_numpy(np.tile(row, (8, 1))).to(G.DEV)
    u = np.array([0.0, -1.0, np.nan, 1.0, 5.0, 0.5, 0.5, 0.5], np.float32)
    tok, prob, kept = run(ctx, logits, u)
    assert tok[:3].tolist() == [0, 0, 0] and tok[3:5].tolist() == [V - 1, V - 1] and (kept == V).all()
    h = np.full(8, 0.37, np.float32)
    T = np.array([np.nan, np.inf, 1e-30, 1e30, 1e-45, 1.0, 1.0, 1.0], np.float32)
    mp = np.array([0, 0, 0, 0, 0, np.nan, 3.0, 0], np.float32)
    p = np.array([1, 1, 1, 1, 1, 1, 1, np.nan], np.float32)
    tok, prob, kept = run(ctx, logits, h, T=T, mp=mp, p=p)
    best, plain = int(np.argmax(row)), PO.sample(row, np.float32(0.37))[0]
    flat = int(0.37 * V)
    assert tok.tolist() == [best, flat, best, flat, best, plain, best, plain]
    assert kept.tolist() == [1, V, V, V, V, V, 1, V] and abs(prob[1] - 1 / V) < 1e-9
    tok, _, kept = run(ctx, logits, h, p=np.full(8, -0.5, np.float32))      # a nucleus of nothing keeps the largest
    assert (tok == best).all() and (kept == 1).all()
    ctx.close()


def test_same_draw_every_time_and_in_a_graph():
    V, n = 16384, 5
    rng = np.random.default_rng(21)
    ctx = make_ctx(V)
    logits = torch.from_numpy(cluster_logits(rng, n, V)).to(G.DEV)
    u, p = dev(rng.random(n), torch.float32), dev(np.full(n, 0.9), torch.float32)
    tok, prob = torch.zeros(n, dtype=torch.int32, device=G.DEV), torch.zeros(n, device=G.DEV)
    cb.cascade_sample(ctx, logits, u, tok, top_p=p, prob=prob)
    first = (tok.clone(), prob.clone())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        cb.cascade_sample(ctx, logits, u, tok, top_p=p, prob=prob)
    for _ in range(5):
        tok.zero_()
        prob.zero_()
        g.replay()
        assert torch.equal(tok, first[0]) and torch.equal(prob, first[1])
    logits.copy_(torch.from_numpy(cluster_logits(rng, n, V)))
    g.replay()
    torch.cuda.synchronize()
    uu = u.cpu().numpy()
    compare(logits, (tok.cpu().numpy(), prob.cpu().numpy(), [PO.sample(logits[r].cpu().numpy(), uu[r], top_p=np.float32(0.9))[2] for r in range(n)]),
            uu, p=np.full(n, 0.9, np.float32))
    ctx.close()


def test_refusals():
    L = cb.lib()
    ctx = make_ctx(64)
    b = torch.zeros(1024, device=G.DEV)
    p = b.data_ptr()

    def call(logits=p, dt=cb.F32, stride=64, n=2, u=p, tok=p + 2048):
        return L.cascade_sample(ctx.handle, logits, dt, stride, n, None, None, None, None, u, tok, None, None, None)
    for bad in (dict(logits=None), dict(dt=7), dict(stride=63), dict(n=0), dict(u=None), dict(tok=None), dict(logits=p + 2)):
        assert call(**bad) == cb.ERR_INVALID_ARG, bad
    assert call(logits=p + 2, dt=cb.BF16) == cb.OK
    ctx.check()
    ctx.close()


def test_arrays_that_are_the_same_are_refused():
    L = cb.lib()
    ctx = make_ctx(64)
    b = torch.zeros(4096, device=G.DEV)
    p = [b.data_ptr() + 1024 * i for i in range(9)]           # logits T k p mp u token prob kept
    def call(a):
        return L.cascade_sample(ctx.handle, a[0], cb.F32, 64, 2, *a[1:], None)
    assert call(p) == cb.OK
    for out in (6, 7, 8):
        for other in range(9):
            if other != out:
                assert call([p[out] if i == other else x for i, x in enumerate(p)]) == cb.ERR_INVALID_ARG, (out, other)
    ctx.check()
    ctx.close()
