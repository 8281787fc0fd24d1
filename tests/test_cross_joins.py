"""The rule of which kernel joins the attention's parts, on the host: the GPU tests' sizes reach each of them behind either
kernel that leaves parts."""
import ctypes
import functools
import os
import random
import subprocess
import tempfile

import test_gpu_cross_attn as A
import test_gpu_cross_joins as J
from test_cross_rules import cross
from test_ffn_tile_rules import CSRC

SHIM = r"""
#include "tile_rules.h"
extern "C" int join(long long rows, int head_dim) { return xema::pick_join(rows, head_dim); }
"""


@functools.lru_cache(None)
def lib():
    with tempfile.TemporaryDirectory(prefix="cross_joins_") as d:
        src, so = os.path.join(d, "shim.cpp"), os.path.join(d, "shim.so")
        with open(src, "w") as f:
            f.write(SHIM)
        subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I" + CSRC, src, "-o", so], check=True)
        return ctypes.CDLL(so)


def join(b, h, d, q):
    return lib().join(ctypes.c_longlong(b * h * q), d)


def joined(sizes):
    """(whether single tokens' kernel left the parts, threads that join a row) of each size in parts"""
    picks = [(cross(*s[:6]), s) for s in sizes]
    return {(few, join(s[0], s[1], s[3], s[4])) for (few, _, parts), s in picks if parts > 1}


def test_sizes_reach_every_join_behind_either_kernel():
    assert joined(A.SIZES + A.TOKENS + J.SIZES) == {(few, threads) for few in (False, True) for threads in (8, 16, 256)}
    assert joined(J.SIZES) == {(few, threads) for few in (False, True) for threads in (8, 16)}


def test_threads_of_a_row_cover_its_head():
    rng = random.Random(4)
    for _ in range(2000):
        rows, d = int(2 ** rng.uniform(0, 24)), 8 * rng.randint(1, 16)
        t = lib().join(ctypes.c_longlong(rows), d)
        assert t == 256 or (t in (8, 16) and 8 * t >= d and rows > 1024)
