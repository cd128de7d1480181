"""cascade_sample at the edges of its settings and of its sums."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as PO
from tests import gpu_util as G
from tests.test_gpu_sample import compare, make_ctx, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,mp", [(np.inf, 0.0), (np.inf, 1e-3), (np.inf, 1.0), (1.0, 0.0), (1.0, 1e-3), (1.0, 1.0), (1e30, 1e-3)])
@pytest.mark.parametrize("p", [1.0, 0.4])
def test_infinite_logits_and_infinite_temperature_with_min_p(T, mp, p):
    V = 264
    rng = np.random.default_rng(2)
    rows = rng.normal(0, 2, (6, V)).astype(np.float32)
    rows[0, [9, 100, 263]] = np.inf
    rows[1, 0] = np.inf
    rows[2, 5:] = np.inf
    rows[3, ::3] = -np.inf
    rows[3, 7] = np.inf
    rows[4, 11] = np.nan
    ctx = make_ctx(V)
    logits = torch.from_numpy(rows).to(G.DEV)
    u = np.array([0.4, 0.9, 0.31, 0.2, 0.613, 0.777], np.float32)
    kw = dict(T=np.full(6, T, np.float32), mp=np.full(6, mp, np.float32), p=np.full(6, p, np.float32))
    # (weights that are exactly min_p = 1, all alike by an infinite temperature, stay: no rounding is near)
    compare(logits, run(ctx, logits, u, **kw), u, gap_min=-1.0 if np.isinf(T) else 1e-9, **kw)
    ctx.close()


def spread(V):
    """How far the fixed-point sums of V weights may be from exact ones, relative to the largest weight: half a unit a weight
    (units of 2^-(62 - log2 V), 2^-50 at the finest) and the weights' own 1e-10."""
    bits = min(50, 62 - int(np.ceil(np.log2(V))))
    return V * 2.0 ** -(bits + 1) + 1e-10


@pytest.mark.parametrize("V", [4096, 65536, 131080, 2 ** 20])
@pytest.mark.parametrize("share", [0.49, 0.51, 3.4])
@pytest.mark.parametrize("p", [None, 0.9999999])
def test_a_flat_tail_at_the_edge_of_the_fixed_point(V, share, p):
    """One logit far above a flat tail whose weights are about half a unit each: all roundings go the same way."""
    bits = min(50, 62 - int(np.ceil(np.log2(V))))
    rng = np.random.default_rng(V)
    n = 6
    x = np.full((n, V), np.log(share * 2.0 ** -bits), np.float32)
    at = rng.integers(0, V, n)
    x[np.arange(n), at] = 0.0
    logits = torch.from_numpy(x).to(G.DEV)
    u = np.array([0.3, 0.999, 1 - 2.0 ** -20, 1 - 2.0 ** -24, 1e-6, 1e-3], np.float32)
    kw = {} if p is None else dict(p=np.full(n, p, np.float32))
    ctx = make_ctx(V)
    tok, prob, kept = run(ctx, logits, u, **kw)
    for r in range(n):
        t, pr, k, gap = PO.sample(logits[r].double().cpu().numpy(), float(u[r]), 1.0, 0, 1.0 if p is None else float(np.float32(p)), 0.0)
        if gap > spread(V):
            assert tok[r] == t and kept[r] == k, (r, gap)
            assert abs(prob[r] - pr) <= spread(V) + 2.0 ** -23 * pr
        else:                                            # on one side of the boundary or on the other
            assert 0 <= tok[r] < V and kept[r] in (1, V)
    ctx.close()
