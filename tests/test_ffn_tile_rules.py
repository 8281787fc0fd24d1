"""The rule by which the feed-forward products pick a tile and a split of k
(csrc/tile_rules.h), on the host: the GPU tests' sizes reach every tile of every
product, and no pick costs more by the rule's own model than another."""
import ctypes
import functools
import os
import random
import subprocess
import tempfile

import test_gpu_ffn as G

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_11136_amd", "csrc")
SHIM = r"""
#include "tile_rules.h"
using namespace xema;
extern "C" {
int count() { return FFN_TILES; }
int pick(long long m, long long n, long long steps) { return pick_tile(m, n, steps); }
int split(long long m, long long n, long long steps, int* parts) {
  const FfnSplit s = pick_split(m, n, steps);
  *parts = s.parts;
  return s.tile;
}
double cost(int t, long long m, long long n, long long steps) { return ffn_tile_us(kFfnCost[t], m, n, steps); }
}
"""


@functools.lru_cache(None)
def lib():
    with tempfile.TemporaryDirectory(prefix="ffn_rules_") as d:
        src, so = os.path.join(d, "shim.cpp"), os.path.join(d, "shim.so")
        with open(src, "w") as f:
            f.write(SHIM)
        subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I" + CSRC, src, "-o", so], check=True)
        out = ctypes.CDLL(so)
        out.cost.restype = ctypes.c_double
        for f in (out.pick, out.split, out.cost):
            f.argtypes = [ctypes.c_int] * (f is out.cost) + [ctypes.c_longlong] * 3 + [ctypes.POINTER(ctypes.c_int)] * (f is out.split)
        return out


def split(m, n, steps):
    parts = ctypes.c_int()
    return lib().split(m, n, steps, ctypes.byref(parts)), parts.value


def test_sizes_reach_every_tile():
    every = set(range(lib().count()))
    steps = lambda k: -(-k // 64)  # noqa: E731
    assert {lib().pick(m, 2 * f, steps(d)) for m, d, f in G.SIZES if m > 32} == every
    assert {lib().pick(m, 2 * f, -(-d // 128)) for m, d, f in G.SIZES_8BIT if m > 32} == every
    assert {lib().pick(m, n, steps(d)) for m, d, n, *_ in G.LORA_SIZES if m > 64 or n > 8192} == every
    assert {lib().pick(2 * f, d, steps(m)) for m, d, f in G.BWD_SIZES} == every
    dx = [split(m, d, 2 * steps(f)) for m, d, f in G.BWD_SIZES]
    assert {t for t, _ in dx} == every and {p for _, p in dx} >= {1, 2, 4, 16}


def test_picks_are_the_cheapest_and_splits_keep_their_bounds():
    rng = random.Random(1)
    for _ in range(3000):
        m, n, steps = (int(2 ** rng.uniform(0, b)) for b in (16, 15, 9))
        costs = [lib().cost(t, m, n, steps) for t in range(lib().count())]
        assert costs[lib().pick(m, n, steps)] == min(costs)
        _, parts = split(m, n, steps)
        assert parts == 1 or (parts <= 16 and steps // parts >= 8 and m * n * parts * 4 <= 64 << 20)
        assert (parts - 1) * -(-steps // parts) < steps      # no part is empty
