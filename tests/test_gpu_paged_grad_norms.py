"""GPU: norms of the paged attention gradient's errors (bounds and their derivation: tests/grad_norms.py), and fp32 products of numbers
whose last bits count."""
import numpy as np
import pytest
import torch

from tests import gpu_util as G
from tests.grad_norms import misses
from tests.test_gpu_paged_grad import Call

pytestmark = pytest.mark.gpu

SHAPES = [([64, 64], [64, 64], 4, 4), ([300], [300], 2, 2), ([640], [640], 2, 1), ([1000], [1000], 1, 1), ([500, 31], [500, 700], 8, 1),
          ([40], [1200], 4, 2), ([2000], [2000], 8, 1), ([129, 257, 385], [640, 257, 900], 10, 2)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("window,sinks", [(0, 0), (100, 3), (512, 0)])
@pytest.mark.parametrize("q_len,kv_len,Hq,Hkv", SHAPES)
def test_norms_of_errors(q_len, kv_len, Hq, Hkv, window, sinks, D, dtype):
    c = Call(q_len, kv_len, Hq, Hkv, D, dtype, window=window, sinks=sinks, seed=41).run()
    for r in range(len(q_len)):
        want, size = c.exact(r)
        for name, x, w, s in zip(("dq", "dk", "dv"), c.got(r), want, size):
            assert misses(dtype, x, w, s) == "", (r, name, misses(dtype, x, w, s))


WORST = 1 + 2.0**-8 - 2.0**-17                                       # bf16 parts 1, 2^-8 and -2^-17


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("carry", ["d_out", "v", "k", "q", "all"])
def test_fp32_products_keep_24_bits(carry, D):
    """One row, one key: P = 1 and dS = <d_out, v>, with one element in each vector.  q or k is zero where the weight is to be exact, so
    that dq and dk come from calls of their own.  A product misses 2^-24 by the terms left out and twice 2^-23 where the tensor cores cut
    sums off (the terms that count are added one by one, the smallest first); dq and dk are two products and a factor, dv is one, all are
    rounded once: 12 2^-24.  Without the last parts 2^-17 = 128 2^-24 is missing."""
    number = lambda name: float(np.float32(WORST)) if carry in (name, "all") else 1.0            # noqa: E731
    for out in ("dq", "dk"):
        c = Call([1], [1], 1, 1, D, "f32", seed=42, scale=0.5)
        for t in (c.q, c.k_pages, c.v_pages, c.d_out):
            t.zero_()
        page = int(c.table_host[0, 0])
        c.d_out[0, 0, 5], c.v_pages[page, 0, 0, 5] = number("d_out"), number("v")
        if out == "dq":
            c.k_pages[page, 0, 0, 9] = number("k")
        else:
            c.q[0, 0, 9] = number("q")
        c.out.zero_()                                                # (delta = 0: the call takes the outputs it is given)
        c.lse.zero_()
        c.backward()
        c.ctx.check()
        g, v, other = number("d_out"), number("v"), number("k" if out == "dq" else "q")
        got = (c.dq if out == "dq" else c.dk)[0, 0].double().cpu().numpy()
        want = np.zeros(D)
        want[9] = 0.5 * g * v * other
        assert np.abs(got - want).max() <= 12 * 2.0**-24 * want[9], (got[9] - want[9]) * 2.0**24
        dv = c.dv[0, 0].double().cpu().numpy()
        dv[5] -= g
        assert np.abs(dv).max() <= 12 * 2.0**-24 * g, dv[5] * 2.0**24


@pytest.mark.parametrize("D", [64, 128])
def test_fp32_scores_keep_24_bits(D):
    """One row, one key, lse = 0: P = exp(c q k) with q k = 1 in parts at their worst: the score is off as above (5 2^-24), its
    argument is rounded twice more (the second time by 2^-24 of 1.44) and the exponential by 2^-22."""
    c = Call([1], [1], 1, 1, D, "f32", seed=43, scale=1.0)
    for t in (c.q, c.k_pages, c.v_pages, c.d_out):
        t.zero_()
    page = int(c.table_host[0, 0])
    c.q[0, 0, 3], c.k_pages[page, 0, 0, 3], c.d_out[0, 0, 5] = WORST, 1.0, 1.0
    c.out.zero_()
    c.lse.zero_()
    c.backward()
    c.ctx.check()
    want = float(np.exp(np.float64(np.float32(WORST))))
    assert abs(float(c.dv[0, 0, 5]) - want) <= (5 + 1 + 1 + 4 + 5) * 2.0**-24 * want
