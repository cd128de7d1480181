"""cascade_sample at the edges of its settings and of its sums."""
import numpy as np
import pytest
import torch

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
