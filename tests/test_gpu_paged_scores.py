"""Scores of minus infinity at keys that a row sees: such a key weighs nothing, and the others decide."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as PO
from tests import gpu_util as G
from tests.test_gpu_paged import Case, half_step, make_ctx

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("q", [1, 9, 150])
@pytest.mark.parametrize("where", [[0], [0, 1, 2], list(range(70)), [5, 64]])
def test_keys_of_infinite_distance(dtype, D, q, where):
    H, page, kv = 2, 16, q + 90
    ctx = make_ctx(dtype, H, H, D)
    c = Case(dtype, H, H, D, page, [q], [kv], seed=q)
    c.q[:, :, 0] = -c.q[:, :, 0].abs() - 0.5                   # times an infinite element: minus infinity
    for x in where:
        c.kp[int(c.table[0, x // page]), x % page, :, 0] = float("inf")
        c.k[0][x, :, 0] = np.inf
    c.run(ctx)
    ctx.check()
    keep = np.setdiff1d(np.arange(kv), where)
    out, lse, qq = (t.double().cpu().numpy() for t in (c.out, c.lse, c.q))
    for i in range(q):
        ok = keep[keep <= kv - q + i]
        ref, ref_lse = PO.attention(qq[i: i + 1], c.k[0][ok], c.v[0][ok], 0, 0, c.scale)
        size, _ = PO.attention(qq[i: i + 1], c.k[0][ok], np.abs(c.v[0][ok]), 0, 0, c.scale)
        tol = (2.0 ** -13 + (2.0 ** -8 if dtype == "bf16" else 0)) * size + half_step(ref, dtype) + 1e-30
        assert (np.abs(out[i: i + 1] - ref) <= tol).all(), i
        assert (np.abs(lse[i: i + 1] - ref_lse) <= 2.0 ** -12 + 2.0 ** -20 * np.abs(ref_lse)).all(), i
    # a value that nobody sees may send rows the long way round: the same outputs
    if q > 1:
        c.vp[int(c.table[0, (kv - 1) // page]), (kv - 1) % page] = float("nan")
        c.run(ctx)
        again = c.out.double().cpu().numpy()
        for i in range(q - 1):
            ok = keep[keep <= kv - q + i]
            ref, _ = PO.attention(qq[i: i + 1], c.k[0][ok], c.v[0][ok], 0, 0, c.scale)
            size, _ = PO.attention(qq[i: i + 1], c.k[0][ok], np.abs(c.v[0][ok]), 0, 0, c.scale)
            tol = (2.0 ** -13 + (2.0 ** -8 if dtype == "bf16" else 0)) * size + half_step(ref, dtype) + 1e-30
            assert (np.abs(again[i: i + 1] - ref) <= tol).all(), i
    ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("q", [1, 40])
def test_rows_all_of_whose_scores_are_minus_infinity_are_no_number(dtype, q):
    ctx = make_ctx(dtype, 2, 2, 64)
    c = Case(dtype, 2, 2, 64, 16, [q], [q + 30])
    c.q[:, :, 0] = -1.0
    c.kp[:, :, :, 0] = float("inf")
    c.run(ctx)
    ctx.check()
    assert torch.isnan(c.out).all()
    ctx.close()
