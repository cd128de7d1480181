"""Bounds for norms of the attention gradient's errors, beside the bounds of single elements, which count every rounding at its worst
and so cannot tell a key more or less in a long row, or 16 bits from 24.

Whole results, |error| <= bound |result| in the sum of squares over a request's dq, dk or dv:

- bf16, 0.003: a number rounded to bf16 is off by 2^-8 / sqrt(12) of its power of two, 0.0016 of itself in the mean square (numbers
  spread evenly over a power of two).  Weights or their gradients are rounded once for a product and the result once, both
  independently: sqrt(2) 0.0016 = 0.0023, and a third more.
- fp32, 2e-6: a weight's argument, at most some 16 in size, is rounded three times: 2^-24 16 / sqrt(12) in the mean square each,
  4.8e-7 together; the exponential is right to 2^-22 (1e-7 in the mean), products of parts and sums of D terms to a few 2^-24
  (1e-7), a weight's gradient, a difference of two numbers a few times its size, to 3e-7: 6e-7 together, and three times that.

Single rows and keys (bf16), |error| <= 2^-6 |row| + 2^-20 |sum of the terms' sizes|: two roundings of at most 2^-8 each, all in one
direction at worst, vectors of 64 elements and more being at right angles but for a third; 32 bits where terms cancel.  A key of average
weight left out of n is an error of n^-1/2: more than that up to 4096 keys."""

WHOLE = {"bf16": 0.003, "f32": 2e-6}
ROW, CANCEL = 2.0**-6, 2.0**-20


def norms(x):
    """Sizes of the rows [.., D] of a result."""
    return (x * x).sum(-1) ** 0.5


def misses(dtype, got, want, size):
    """What of one result (64-bit arrays or tensors [.., D]) lies outside the bounds: '' or a description."""
    error, whole = norms(got - want), norms(want)
    e, w = float((error ** 2).sum() ** 0.5), float((whole ** 2).sum() ** 0.5)
    if not e <= WHOLE[dtype] * w:
        return f"error {e / max(w, 1e-300):.2e} of the whole"
    if dtype == "bf16":
        over = error - (ROW * whole + CANCEL * norms(size))
        if not float(over.max()) <= 0:
            return f"a row off by {float((error / (whole + 1e-300)).max()):.2e} of itself"
    return ""
