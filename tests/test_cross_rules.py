"""The launchers' rules of the cross-attention sub-block (csrc/tile_rules.h) on the
host: the GPU tests' sizes reach every kernel, whole and in parts, and parts stay
within what the kernels and the workspace allow."""
import ctypes
import functools
import os
import random
import subprocess
import tempfile

import test_gpu_cross_attn as A
import test_gpu_linear as L
from test_ffn_tile_rules import CSRC, lib as tiles, split
from test_ffn_variants import pick, steps

SHIM = r"""
#include "tile_rules.h"
using namespace xema;
extern "C" {
int cross(int batch, int heads, int kv_heads, int head_dim, int q_len, int kv_len, int* blocks, int* parts) {
  const CrossPick p = pick_cross(batch, heads, kv_heads, head_dim, q_len, kv_len);
  *blocks = p.blocks;
  *parts = p.parts;
  return p.few;
}
int rows(long long m, long long n, long long steps, long long* first) {
  const FfnRows p = pick_rows(m, n, steps);
  *first = p.rows;
  return p.rest;
}
int bwd(int batch, int heads, int kv_heads, int head_dim, int q_len, int kv_len, int* q_parts, int* kv_parts) {
  const CrossBwdPick p = pick_cross_bwd(batch, heads, kv_heads, head_dim, q_len, kv_len);
  *q_parts = p.q_parts;
  *kv_parts = p.kv_parts;
  return p.both;
}
}
"""


@functools.lru_cache(None)
def lib():
    with tempfile.TemporaryDirectory(prefix="cross_rules_") as d:
        src, so = os.path.join(d, "shim.cpp"), os.path.join(d, "shim.so")
        with open(src, "w") as f:
            f.write(SHIM)
        subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I" + CSRC, src, "-o", so], check=True)
        return ctypes.CDLL(so)


def cross(b, h, kh, d, q, kv):
    blocks, parts = ctypes.c_int(), ctypes.c_int()
    few = lib().cross(b, h, kh, d, q, kv, ctypes.byref(blocks), ctypes.byref(parts))
    return bool(few), blocks.value, parts.value


def bwd(b, h, kh, d, q, kv):
    q_parts, kv_parts = ctypes.c_int(), ctypes.c_int()
    both = lib().bwd(b, h, kh, d, q, kv, ctypes.byref(q_parts), ctypes.byref(kv_parts))
    return bool(both), q_parts.value, kv_parts.value


def rows(m, n, steps):
    first = ctypes.c_longlong()
    size = [ctypes.c_longlong(x) for x in (m, n, steps)]
    return lib().rows(*size, ctypes.byref(first)), first.value


def width(d):
    return -(-d // 32)


def test_linear_sizes_reach_every_tile_and_few_row_kernel():
    few = {(m, d, n): pick("lora_few", m, n) for m, d, n in L.SIZES}
    assert set(few.values()) == {(r, c) for c in (1, 2) for r in (1, 2, 3, 4)} | {(1, 4), (2, 4), (0, 0)}
    found = {rows(m, n, steps(d)) for (m, d, n), p in few.items() if p == (0, 0)}
    assert {t for t, _ in found} == set(range(tiles().count())) and {first > 0 for _, first in found} == {False, True}


def test_rows_of_a_launch_of_their_own():
    """A multiple of 256 with something left, where the rule's model says that the two launches take less."""
    rng = random.Random(2)
    split_some = 0
    for _ in range(3000):
        m, n, k = (int(2 ** rng.uniform(0, b)) for b in (16, 15, 9))
        tile, first = rows(m, n, k)
        assert first % 256 == 0 and 0 <= first < m
        whole = min(tiles().cost(t, m, n, k) for t in range(tiles().count()))
        if first:
            split_some += 1
            assert tiles().cost(0, first, n, k) + 3 + tiles().cost(tile, m - first, n, k) < whole
        else:
            assert tiles().cost(tile, m, n, k) == whole
    assert split_some > 100


def test_linear_gradients_reach_every_tile_whole_and_split():
    dx, dw = {split(m, d, steps(n)) for m, d, n in L.BWD_SIZES}, {split(n, d, steps(m)) for m, d, n in L.BWD_SIZES}
    assert {(t, parts > 1) for t, parts in dx | dw} == {(t, s) for t in range(5) for s in (False, True)}
    for found in (dx, dw):
        assert {parts > 1 for _, parts in found} == {False, True}
    assert {split(m, d, steps(n))[0] == split(n, d, steps(m))[0] for m, d, n in L.BWD_SIZES} == {False, True}


def test_attention_sizes_reach_every_kernel_whole_and_in_parts():
    sizes = [s[:6] for s in A.SIZES + A.TOKENS]
    found = {(width(s[3]), cross(*s)[0], cross(*s)[2] > 1) for s in sizes}
    assert found >= {(w, few, False) for w in (1, 2, 3, 4) for few in (False, True)}
    assert found >= {(w, True, True) for w in (1, 2, 3, 4)} | {(w, False, True) for w in (1, 2, 3, 4)}
    sizes = [s[:6] for s in A.SIZES + A.TOKENS[1:6]]
    found = {(width(s[3]), *bwd(*s)) for s in sizes}
    assert {(w, both, parts > 1) for w, both, parts, _ in found} >= {(w, True, p) for w in (1, 2, 3, 4) for p in (False, True)}
    assert {(w, both, parts > 1) for w, both, _, parts in found} >= {(w, b, p) for w in (1, 2, 3, 4) for b in (False, True) for p in (False, True)}


def test_parts_stay_in_bounds():
    rng = random.Random(1)
    for _ in range(20000):
        kh, group, d = rng.randint(1, 64), rng.choice((1, 1, 2, 8, 32)), 8 * rng.randint(1, 16)
        b, q, kv = int(2 ** rng.uniform(0, 12)), int(2 ** rng.uniform(0, 20)), int(2 ** rng.uniform(0, 20)) - 1
        h = kh * group
        few, blocks, parts = cross(b, h, kh, d, q, kv)
        assert 1 <= parts <= 64 and blocks >= 1
        assert parts == 1 or parts <= -(-kv // 32)
        per = 32 if few else 128
        assert (blocks - 1) * per < q * (group if few else 1) <= blocks * per
        if parts > 1:      # the sums of all parts stay within 512 MiB
            assert parts * b * h * q * (4 * d + 8) < 1 << 29
        both, dq, dkv = bwd(b, h, kh, d, q, kv)
        assert 1 <= dq <= 16 and (dq == 1 or dq * b * h * q * d * 4 < 1 << 29)
        assert 1 <= dkv <= 32 and (dkv == 1 or dkv * 2 * b * kv * kh * d <= 1 << 26)
        assert not both or b * h * -(-q // 128) * dq + b * kh * -(-kv // 128) * dkv <= 512
