"""Whether two arguments of a feed-forward entry point overlap (csrc/spans.h),
on the host, against the sets of their bytes."""
import ctypes
import functools
import os
import random
import subprocess
import tempfile

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_11136_amd", "csrc")
SHIM = r"""
#include "spans.h"
using namespace xema;
extern "C" int meet(long long a, long long aw, long long ar, long long ap, long long b, long long bw, long long br, long long bp) {
  return overlaps(span_rows((const void*)a, aw, ar, ap), span_rows((const void*)b, bw, br, bp));
}
"""


@functools.lru_cache(None)
def lib():
    with tempfile.TemporaryDirectory(prefix="ffn_spans_") as d:
        src, so = os.path.join(d, "shim.cpp"), os.path.join(d, "shim.so")
        with open(src, "w") as f:
            f.write(SHIM)
        subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-shared", "-fPIC", "-I" + CSRC, src, "-o", so], check=True)
        out = ctypes.CDLL(so)
        out.meet.argtypes = [ctypes.c_longlong] * 8
        return out


def meet(a, b):
    one, other = lib().meet(*a, *b), lib().meet(*b, *a)
    assert one == other
    return bool(one)


def bytes_of(p, width, rows, pitch):
    return {p + r * pitch + c for r in range(rows) for c in range(width)}


def test_against_the_sets_of_bytes():
    rng = random.Random(1)
    seen = set()
    for _ in range(20000):
        pitch = rng.randint(1, 24)
        a = (1000, rng.randint(1, pitch), rng.randint(0, 6), pitch)
        kind = rng.choice(("same pitch", "vector"))
        w, rows, p = (rng.randint(1, pitch), rng.randint(0, 6), pitch) if kind == "same pitch" else (rng.randint(1, 60), 1, 60)
        b = (1000 + rng.randint(-150, 150), w, rows, p)
        want = bool(bytes_of(*a) & bytes_of(*b))
        assert meet(a, b) == want, (a, b)
        seen.add((kind, want))
    assert len(seen) == 4


def test_unlike_pitches_never_miss_an_overlap():
    rng = random.Random(2)
    for _ in range(5000):
        a, b = ((1000 + rng.randint(-60, 60), rng.randint(1, 9), rng.randint(1, 6), rng.randint(9, 30)) for _ in range(2))
        assert meet(a, b) or not bytes_of(*a) & bytes_of(*b)


def test_sizes_of_real_arguments():
    n, pitch = (1 << 24) - 1, ((1 << 21) - 8) * 4
    x = (1 << 40, 4096, n, pitch)
    assert not meet(x, ((1 << 40) + 4096, 4096, n, pitch))            # the next columns of the same buffer
    assert meet(x, ((1 << 40) + 4095, 4096, n, pitch))
    assert not meet(x, ((1 << 40) + n * pitch, 4096, n, pitch)) and not meet(x, ((1 << 40) - n * pitch, 4096, n, pitch))
    assert meet(x, ((1 << 40) - (n - 1) * pitch, 4096, n, pitch))
    assert not meet(x, ((1 << 40) + 4096, 64, 1, 64)) and meet(x, ((1 << 40) + pitch - 4, 64, 1, 64))
    assert not meet((0, 64, 4, 64), (0, 64, 4, 64)) and not meet(x, (1 << 40, 64, 0, 64))     # null, no rows
