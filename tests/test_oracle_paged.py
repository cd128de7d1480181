"""Pins of the 64-bit restatements of the paged calls and sampling (CPU), and of the calls' host-side refusals."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from oracle import paged_oracle as PO
from paper_2605_07230_b200 import binding as cb


@pytest.mark.parametrize("n,kv,Hq,Hkv,D", [(5, 5, 4, 4, 8), (3, 11, 6, 2, 16), (1, 1, 1, 1, 8)])
def test_attention_is_the_causal_softmax(n, kv, Hq, Hkv, D):
    rng = np.random.default_rng(0)
    q, k, v = rng.normal(size=(n, Hq, D)), rng.normal(size=(kv, Hkv, D)), rng.normal(size=(kv, Hkv, D))
    out, lse = PO.attention(q, k, v, 0, 0, 0.3)
    rep = lambda t: torch.from_numpy(t).repeat_interleave(Hq // Hkv, 1).transpose(0, 1)  # noqa: E731
    mask = torch.ones(n, kv).tril(kv - n).bool()
    ref = torch.nn.functional.scaled_dot_product_attention(torch.from_numpy(q).transpose(0, 1), rep(k), rep(v),
                                                           attn_mask=mask, scale=0.3).transpose(0, 1)
    assert np.allclose(out, ref.numpy(), atol=1e-12)
    s = (torch.from_numpy(q).transpose(0, 1) @ rep(k).transpose(1, 2) * 0.3).masked_fill(~mask, -math.inf)
    assert np.allclose(lse.T, torch.logsumexp(s, -1).numpy(), atol=1e-12)


def test_window_and_sinks_by_hand():
    assert PO.sees(5, 8, 0, 0).tolist() == [True] * 6 + [False] * 2
    assert PO.sees(5, 8, 2, 0).tolist() == [False] * 4 + [True] * 2 + [False] * 2
    assert PO.sees(5, 8, 2, 1).tolist() == [True, False, False, False, True, True, False, False]
    assert PO.sees(5, 8, 100, 3).tolist() == [True] * 6 + [False] * 2
    assert not PO.sees(-1, 4, 3, 2).any()
    out, lse = PO.attention(np.ones((3, 1, 4)), np.ones((1, 1, 4)), np.ones((1, 1, 4)), 0, 0, 1.0)   # two rows see nothing
    assert (out[:2] == 0).all() and np.isneginf(lse[:2]).all() and (out[2] == 1).all()


def test_rotation_keeps_norms_and_relative_positions():
    rng = np.random.default_rng(1)
    x, y = rng.normal(size=(1, 2, 16)), rng.normal(size=(1, 2, 16))
    for p in (0, 3, 70000):
        a, b = PO.rotate(x, [p + 5], 1e4), PO.rotate(y, [p], 1e4)
        assert np.allclose((a * b).sum(-1), (PO.rotate(x, [5], 1e4) * y).sum(-1), atol=1e-9)
        assert np.allclose((a * a).sum(-1), (x * x).sum(-1))
    assert np.array_equal(PO.rotate(x, [0], 1e4), x)


def test_tables_walk_by_hand():
    #  request 0: 5 tokens in one page of 8, takes 4 (one more page); 1: finished, 9 tokens (pages 4, 2); 2: empty, takes 8
    table = [[7, -1, -1], [4, 2, -1], [-1, -1, -1]]
    got = PO.tables([4, -1, 8], [5, 9, 0], table, [3, 6, 0, 0, 0, 0, 0, 0], 2, 8, 14)
    assert got["table"].tolist() == [[7, 2, -1], [4, 2, -1], [4, -1, -1]]     # 2 was pushed last, then 4
    assert got["count"] == 2 and got["free"][:2].tolist() == [3, 6] and got["kv"].tolist() == [9, 0, 8]
    assert got["q_begin"].tolist() == [0, 4, 4, 12]
    assert got["slot"].tolist() == [61, 62, 63, 16] + list(range(32, 40)) + [-1, -1]
    assert got["pos"].tolist() == [5, 6, 7, 8] + list(range(8)) + [-1, -1]
    assert PO.tables([30, 0, 0], [5, 0, 0], table, [3, 6] + [0] * 6, 2, 8, 99) is None       # wider than the table
    assert PO.tables([4, 8, 17], [5, 9, 0], table, [3, 6] + [0] * 6, 2, 8, 99) is None       # needs more pages than there are
    assert PO.tables([4, -1, 8], [5, 9, 0], table, [3, 6] + [0] * 6, 2, 8, 11) is None       # more tokens than rows


def test_sampling_covers_the_distribution():
    rng = np.random.default_rng(2)
    row = rng.normal(size=11)
    row[3] = -np.inf
    row[5] = np.nan
    us = (np.arange(20000) + 0.5) / 20000
    p = np.exp(np.where(np.isfinite(row), row, -np.inf) / 0.7)
    p /= p.sum()
    draws = np.bincount([PO.sample(row, u, 0.7)[0] for u in us], minlength=11) / 20000
    assert np.abs(draws - p).max() < 1e-4
    for k, pp, mp in ((3, 1.0, 0.0), (0, 0.5, 0.0), (0, 1.0, 0.3), (6, 0.8, 0.2)):
        order = np.argsort(-np.where(np.isfinite(row), row, -np.inf), kind="stable")
        keep = np.zeros(11, bool)
        keep[order[: k or 9]] = True
        if pp < 1:
            q = np.where(keep, p, 0) / p[keep].sum()
            before = np.concatenate([[0], np.cumsum(q[order])[:-1]])
            keep[order[before >= pp]] = False
        keep &= p >= mp * p.max()
        t, prob, kept, _ = PO.sample(row, 0.4, 0.7, k, pp, mp)
        assert kept == keep.sum() and keep[t] and math.isclose(prob, p[t] / p[keep].sum())
    assert PO.sample([1.0, 2.0, 2.0], 0.9, 0.0)[:3] == (1, 1.0, 1)
    assert PO.sample([-np.inf, np.nan], 0.9)[:3] == (-1, 0.0, 0)
    assert PO.sample([1.0, np.inf, 0.0, np.inf], 0.6)[:3] == (3, 0.5, 4)


def test_null_contexts_are_refused_without_a_device():
    L = cb.lib()
    assert L.cascade_paged_tables(None, 1, 1, 8, 1, None, None, None, 1, None, None, None, None, None, None, None, None) == cb.ERR_INVALID_ARG
    assert L.cascade_paged_append(None, None, 1, None, 0, None, 0, None, 0, None, None, 0.0, None, 0, None) == cb.ERR_INVALID_ARG
    assert L.cascade_paged_attn(None, None, 1, 1, None, 0, None, None, 1, 1, 0, 0, 1.0, None, None, None) == cb.ERR_INVALID_ARG
    assert L.cascade_sample(None, None, 0, 1, 1, None, None, None, None, None, None, None, None, None) == cb.ERR_INVALID_ARG
    assert b"page" in L.cascade_strerror(cb.ERR_BAD_PAGE)
    assert C.sizeof(cb.PagedCacheStruct) == 48


class _FakeCtx:
    """What the binding looks at before it calls the library."""

    def __init__(self, dtype=cb.BF16, Hq=4, Hkv=2, D=64, V=64):
        self.shape, self.handle = cb.Shape(dtype, 1, 1, 64, 64, Hq, Hkv, D, V, 0), None


def test_binding_refuses_wrong_tensors():
    ctx = _FakeCtx()
    bf, i32 = torch.bfloat16, torch.int32
    pool = torch.zeros(3, 8, 2, 64, dtype=bf)
    table = torch.zeros(1, 3, dtype=i32)
    cache = cb.PagedCache(pool, pool.clone(), table)
    k = torch.zeros(5, 2, 64, dtype=bf)
    idx = torch.zeros(5, dtype=i32)
    q = torch.zeros(5, 4, 64, dtype=bf)
    for bad in (lambda: cb.PagedCache(pool, pool.float(), table),
                lambda: cb.PagedCache(pool, pool[:2], table),
                lambda: cb.PagedCache(pool.transpose(1, 2), pool.transpose(1, 2), table),
                lambda: cb.PagedCache(pool, pool, table.long()),
                lambda: cb.PagedCache(pool, pool, table.T),
                lambda: cb.cascade_paged_append(ctx, cache, k.float(), k, idx, idx),
                lambda: cb.cascade_paged_append(ctx, cache, k[:4], k, idx, idx),
                lambda: cb.cascade_paged_append(ctx, cache, k, k, idx.long(), idx),
                lambda: cb.cascade_paged_append(ctx, cache, k.transpose(1, 2).contiguous().transpose(1, 2), k, idx, idx),
                lambda: cb.cascade_paged_append(_FakeCtx(D=128), cache, k, k, idx, idx),
                lambda: cb.cascade_paged_attn(ctx, cache, q, idx, idx, 1, 1, q, 1.0),
                lambda: cb.cascade_paged_attn(ctx, cache, q, idx[:3], idx[:2], 1, 1, q, 1.0),     # two requests, one table row
                lambda: cb.cascade_paged_attn(ctx, cache, q, idx[:2], idx[:1], 1, 1, q[:4], 1.0),
                lambda: cb.cascade_paged_attn(_FakeCtx(cb.F32), cache, q, idx[:2], idx[:1], 1, 1, q, 1.0),
                lambda: cb.cascade_sample(ctx, torch.zeros(5, 32), torch.zeros(5), idx),
                lambda: cb.cascade_sample(ctx, torch.zeros(5, 64).half(), torch.zeros(5), idx),
                lambda: cb.cascade_sample(ctx, torch.zeros(64, 5).T, torch.zeros(5), idx),
                lambda: cb.cascade_sample(ctx, torch.zeros(5, 64), torch.zeros(4), idx),
                lambda: cb.cascade_sample(ctx, torch.zeros(5, 64), torch.zeros(5), idx, top_k=torch.zeros(5)),
                lambda: cb.cascade_paged_tables(ctx, 8, 3, idx, idx, table, idx[:3], idx[:1], idx, idx[:1], idx, idx, idx)):
        with pytest.raises(ValueError) as e:
            bad()
        assert "current CUDA device" not in str(e.value)
    for off_device in (lambda: cb.cascade_paged_append(ctx, cache, k, k, idx, idx),          # all right but for where they live
                       lambda: cb.cascade_sample(ctx, torch.zeros(5, 64), torch.zeros(5), idx)):
        with pytest.raises(ValueError, match="current CUDA device"):
            off_device()
