"""The bounds of tests/grad_norms.py tell apart what they are for (CPU): the gradient with its roundings as the library makes them
lies inside, a key left out, parts left out of a 32-bit number, or a 16-bit operand too many lie outside."""
import numpy as np
import pytest

from oracle import train_oracle as TO
from tests.grad_norms import misses


def bf16(x):
    """Nearest bf16, ties to even, of 32-bit numbers in 64 bits."""
    u = np.asarray(x, np.float32).view(np.uint32).astype(np.uint64)
    u = (u + 0x7FFF + ((u >> 16) & 1)) & 0xFFFF0000
    return u.astype(np.uint32).view(np.float32).astype(np.float64)


def parts(x, n):
    out, x = [], np.asarray(x, np.float32).astype(np.float64)
    for _ in range(n):
        out.append(bf16(x))
        x = x - out[-1]
    return out


def product(spec, a, b, n):
    """A product of 32-bit numbers as n bf16 parts each: the terms from hh down to the n-th order."""
    pa, pb = parts(a, n), parts(b, n)
    return sum(np.einsum(spec, pa[i], pb[j]) for i in range(n) for j in range(n) if i + j < n)


def attention(rng, n, kv, H, D, window):
    """Inputs, what the forward pass leaves, and the mask."""
    q, g = rng.standard_normal((2, n, H, D)).astype(np.float32)
    k, v = rng.standard_normal((2, kv, H, D)).astype(np.float32)
    x, j = (kv - n + np.arange(n))[:, None], np.arange(kv)[None]
    see = (j <= x) & ((j > x - window) if window else True)
    return q, k, v, g, see


def forward(q, k, v, see, scale, rounded):
    s = np.where(see[None], np.einsum("ihd,jhd->hij", q, k) * scale, -np.inf)
    lse = np.log(np.exp(s - s.max(-1, keepdims=True)).sum(-1)) + s.max(-1)
    out = np.einsum("hij,jhd->ihd", np.exp(s - lse[..., None]), v)
    return rounded(out), lse.astype(np.float32).astype(np.float64)


def gradient(q, k, v, g, see, out, lse, scale, times, operand, result):
    """The formulas with products by `times`, operands of the second products and results rounded."""
    p = np.where(see[None], np.exp(times("ihd,jhd->hij", q, k) * scale - lse[..., None]), 0.0)
    ds = p * (times("ihd,jhd->hij", g, v) - (g.astype(np.float64) * out).sum(-1).T[..., None])
    p, ds = operand(p), operand(ds)
    return [result(x) for x in (scale * times("hij,jhd->ihd", ds, k), scale * times("hij,ihd->jhd", ds, q), times("hij,ihd->jhd", p, g))]


SHAPES = [(64, 64, 0), (300, 300, 0), (40, 700, 0), (500, 600, 100)]


@pytest.mark.parametrize("n,kv,window", SHAPES)
def test_bf16_roundings_and_a_key_left_out(n, kv, window):
    rng = np.random.default_rng(n)
    D, scale = 64, 0.125
    q, k, v, g, see = attention(rng, n, kv, 1, D, window)
    q, k, v, g = (bf16(t) for t in (q, k, v, g))
    out, lse = forward(q, k, v, see, scale, bf16)
    want, size = TO.attention_grad(q, k, v, g, window, 0, scale, out=out, lse=lse.T)
    plain = lambda spec, a, b: np.einsum(spec, a, b)                                             # noqa: E731
    got = gradient(q, k, v, g, see, out, lse, scale, plain, bf16, bf16)
    assert [misses("bf16", *t) for t in zip(got, want, size)] == ["", "", ""]
    # one key of one row in the middle, a key that the rows at its tile's end do not get, the window one key short
    row = see.copy()
    row[n // 2, kv - n // 2 - 8] = False
    tile = see.copy()
    tile[-(n // 4):, (kv // 2) // 128 * 128] = False
    short = see.copy()
    short[np.arange(n), np.maximum(0, kv - n + np.arange(n) - (window or kv) + 1)] = False
    for spoiled in (row, tile, short):
        bad = gradient(q, k, v, g, spoiled, out, lse, scale, plain, bf16, bf16)
        where = [misses("bf16", *t) for t in zip(bad, want, size)]
        assert (spoiled == see).all() or any(where), where


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n,kv,window", SHAPES)
def test_three_parts_of_a_32_bit_number_and_two(n, kv, window, D):
    rng = np.random.default_rng(n + D)
    scale = D**-0.5
    q, k, v, g, see = attention(rng, n, kv, 1, D, window)
    single = lambda x: np.asarray(x, np.float32).astype(np.float64)                              # noqa: E731
    out, lse = forward(*(t.astype(np.float64) for t in (q, k, v)), see, scale, single)
    want, size = TO.attention_grad(q, k, v, g, window, 0, scale, out=out, lse=lse.T)
    by_parts = lambda m: lambda spec, a, b: product(spec, a, b, m)                               # noqa: E731
    for m, inside in ((3, True), (2, False), (1, False)):
        got = gradient(q, k, v, g, see, out, lse, scale, by_parts(m), single, single)
        for t in zip(got, want, size):
            assert (misses("f32", *t) == "") == inside, (m, misses("f32", *t))


def test_parts_at_their_worst():
    """1 + 2^-8 - 2^-17 has parts of 1, 2^-8 and -2^-17: the terms left out of a square are nearly 2^-24 of it."""
    x = np.float32(1 + 2.0**-8 - 2.0**-17)
    assert [float(p) for p in parts(x, 3)] == [1.0, 2.0**-8, -(2.0**-17)]
    exact = float(x) ** 2
    assert 0.9 * 2.0**-24 < abs(float(product(",->", x, x, 3)) - exact) / exact < 2.0**-24
    # beside a power of two every part counts: three are the number, two miss 2^-17 of it
    three, two = (float(product(",->", x, np.float32(1), m)) for m in (3, 2))
    assert three == float(x) and abs(two - float(x)) > 100 * 2.0**-24
