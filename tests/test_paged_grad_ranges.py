"""Which rows see a tile of keys, in the attention's gradient: the kernels' own arithmetic, compiled for the host, against integers of
any size (lengths that no test can hold)."""
import os
import random
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2605_07230_b200", "csrc")
PROGRAM = r"""
#include <cstdio>
#include "paged_range.h"
struct Args { int window, sinks; };
int main() {
  Args a;
  int x0, nq, G, first, last, lo, hi;
  while (std::scanf("%d %d %d %d %d %d %d", &a.window, &a.sinks, &x0, &nq, &G, &first, &last) == 7) {
    paged::rows_that_see(a, x0, nq, G, first, last, &lo, &hi);
    std::printf("%d %d\n", lo, hi);
  }
}
"""
MOST = 2**31 - 65536                                                 # keys of a request, and rows of a key head


def cases():
    rng = random.Random(1)
    up_to = lambda n: min(n, int(2 ** rng.uniform(0, 31)))           # noqa: E731
    # a window that ends far in front of the new tokens, many query heads a key head: 2^24 keys and more
    yield from [(64, 0, 20_000_000, 5, 128, 0, 127), (1, 4, MOST - 3, 3, 128, 128, 255), (1000, 0, 17_000_000, 300, 128, 384, 511),
                (2**31 - 1, 0, MOST - 9, 9, 100, 0, 127), (64, 100, 20_000_000, 5, 128, 128, 255), (64, 200, 20_000_000, 5, 128, 128, 255)]
    for _ in range(4000):
        G = rng.choice([1, 2, 5, 8, 100, 128])
        nq = up_to(MOST // G)
        kv = rng.choice([max(1, nq - up_to(nq)), max(1, min(MOST, nq + up_to(MOST)))])
        first = rng.randrange(0, kv) // 128 * 128
        yield (rng.choice([0, up_to(2**31 - 1)]), rng.choice([0, 4, up_to(2**31 - 1)]), kv - nq, nq, G, first, min(first + 127, kv - 1))


def seen(window, sinks, x0, nq, G, first, last):
    """Tokens t with a key j of the range: j <= x0 + t, and j inside the window or among the first ones."""
    lo, hi = max(0, first - x0), nq
    if window and first >= sinks:
        hi = min(nq, last + window - x0)
    return lo * G, hi * G


@pytest.mark.skipif(shutil.which("g++") is None, reason="no host compiler")
def test_rows_that_see_a_tile_of_keys(tmp_path):
    (tmp_path / "main.cpp").write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-ftrapv", "-I" + CSRC, str(tmp_path / "main.cpp"), "-o", str(tmp_path / "main")], check=True)
    want = list(cases())
    text = "\n".join(" ".join(map(str, c)) for c in want)
    r = subprocess.run([str(tmp_path / "main")], input=text, capture_output=True, text=True)
    got = [tuple(map(int, line.split())) for line in r.stdout.splitlines()]
    assert r.returncode == 0 and len(got) == len(want), (len(got), want[len(got)] if len(got) < len(want) else None)
    for c, (lo, hi) in zip(want, got):
        a, b = seen(*c)
        rows = c[3] * c[4]
        if a >= b:                                                   # nobody: an empty range inside the request's rows
            assert 0 <= hi <= lo <= rows, (c, lo, hi)
        else:
            assert (lo, hi) == (a, b) and 0 <= lo < hi <= rows, (c, lo, hi)


def test_the_range_is_that_of_the_definition():
    rng = random.Random(2)
    for _ in range(500):
        window, sinks, nq, kv = rng.choice([0, rng.randint(1, 30)]), rng.choice([0, rng.randint(0, 30)]), rng.randint(1, 30), rng.randint(1, 40)
        first = rng.randrange(kv)
        last = rng.randrange(first, min(kv, first + 9))
        x0 = kv - nq
        ok = [t for t in range(nq) if any(j <= x0 + t and (window == 0 or j > x0 + t - window or j < sinks) for j in range(first, last + 1))]
        lo, hi = seen(window, sinks, x0, nq, 1, first, last)
        assert ok == list(range(lo, hi)), (window, sinks, nq, kv, first, last)
