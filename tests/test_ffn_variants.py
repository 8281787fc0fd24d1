"""The launchers' rules (csrc/tile_rules.h) on the host: the GPU tests' sizes
reach every tile with and without a split of k, every block of the adapters'
reduction and every few-row kernel, counted as the launchers choose them."""
import ctypes
import functools
import os
import subprocess
import tempfile

import test_gpu_ffn as G
import test_gpu_ffn_variants as V
from test_ffn_tile_rules import CSRC, lib as tiles, split

SHIM = r"""
#include "tile_rules.h"
using namespace xema;
extern "C" {
int reduce_blocks(long long rows, int rank) { const ReducePick p = pick_reduce(rows, rank); return p.rows16 * 10 + p.ranks16; }
int lora_few(long long rows, int out_dim) { const FewPick p = pick_lora_few(rows, out_dim); return p.rows16 * 10 + p.cols16; }
int gated_few(long long rows, int hidden) { const FewPick p = pick_gated_few(rows, hidden); return p.rows16 * 10 + p.cols16; }
}
"""


@functools.lru_cache(None)
def lib():
    with tempfile.TemporaryDirectory(prefix="ffn_variants_") as d:
        src, so = os.path.join(d, "shim.cpp"), os.path.join(d, "shim.so")
        with open(src, "w") as f:
            f.write(SHIM)
        subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I" + CSRC, src, "-o", so], check=True)
        out = ctypes.CDLL(so)
        for f in (out.reduce_blocks, out.lora_few, out.gated_few):
            f.argtypes = [ctypes.c_longlong, ctypes.c_int]
        return out


def pick(rule, *args):
    return divmod(getattr(lib(), rule)(*args), 10)


def steps(k):
    return -(-k // 64)


TILES = range(5)


def test_gradients_reach_every_tile_whole_and_split():
    assert tiles().count() == len(TILES)
    sizes = G.BWD_SIZES + V.BWD_SIZES
    both = {(t, s) for t in TILES for s in (False, True)}
    for found in ({split(2 * f, d, steps(m)) for m, d, f in sizes}, {split(m, d, 2 * steps(f)) for m, d, f in sizes}):
        assert {(t, parts > 1) for t, parts in found} == both
    # one launch for both products, and one each
    assert {split(2 * f, d, steps(m))[0] == split(m, d, 2 * steps(f))[0] for m, d, f in sizes} == {False, True}


def test_forward_sizes_reach_every_tile_and_few_row_kernel():
    for sizes, kb in ((G.SIZES, 64), (G.SIZES_8BIT, 128)):
        few = {(m, d, f): pick("gated_few", m, f) for m, d, f in sizes}
        assert set(few.values()) == {(1, 1), (2, 1), (0, 0)}
        assert {tiles().pick(m, 2 * f, -(-d // kb)) for (m, d, f), p in few.items() if p == (0, 0)} == set(TILES)


def test_projections_reach_every_tile_few_row_kernel_and_reduction():
    sizes = G.LORA_SIZES + V.LORA_SIZES
    few = {(m, d, n): pick("lora_few", m, n) for m, d, n, *_ in sizes}
    assert set(few.values()) == {(r, c) for c in (1, 2) for r in (1, 2, 3, 4)} | {(1, 4), (2, 4), (0, 0)}
    assert {tiles().pick(m, n, steps(d)) for (m, d, n), p in few.items() if p == (0, 0)} == set(TILES)
    assert {pick("reduce_blocks", m, r) for m, _, _, r, _ in sizes} == {(m, r) for m in (1, 2, 3) for r in (1, 2, 4)} | {(0, 0)}


def test_reductions_give_every_cu_a_workgroup_where_they_can():
    for rank in range(8, 129, 8):
        for rows in [*range(1, 600), 1000, 2000, 4096, 4097, 8000, 12288, 12289, 50000, (1 << 24) - 1]:
            m, r = pick("reduce_blocks", rows, rank)
            if m == 0:
                assert rows * rank <= 32768
                continue
            assert rows * rank > 32768 and m in (1, 2, 3) and r in (1, 2, 4)
            assert r == 1 or (rank > 8 * r and -(-rows // (16 * m)) * -(-rank // (16 * r)) >= 256)
            assert m == 1 or -(-rows // (16 * m)) >= 256 or rows > 16 * 256
