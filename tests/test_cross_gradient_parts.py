"""The launches of dk and dv without dq, on the host: the pass that leaves lse and D goes over the tokens once."""
import ctypes
import functools
import os
import random
import subprocess
import tempfile

from test_cross_rules import bwd
from test_ffn_tile_rules import CSRC

SHIM = r"""
#include "tile_rules.h"
using namespace xema;
extern "C" int alone(int batch, int heads, int kv_heads, int head_dim, int q_len, int kv_len, int* q_parts, int* kv_parts) {
  const CrossBwdPick p = without_dq(pick_cross_bwd(batch, heads, kv_heads, head_dim, q_len, kv_len));
  *q_parts = p.q_parts;
  *kv_parts = p.kv_parts;
  return p.both;
}
"""


@functools.lru_cache(None)
def lib():
    with tempfile.TemporaryDirectory(prefix="cross_gradient_parts_") as d:
        src, so = os.path.join(d, "shim.cpp"), os.path.join(d, "shim.so")
        with open(src, "w") as f:
            f.write(SHIM)
        subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I" + CSRC, src, "-o", so], check=True)
        return ctypes.CDLL(so)


def test_tokens_are_met_once_without_dq():
    rng = random.Random(6)
    split = 0
    for size in [(1, 8, 8, 128, 128, 4096), (1, 8, 8, 128, 20, 4000)] + [
            (rng.randint(1, 4), 8, rng.choice((1, 2, 8)), 8 * rng.randint(1, 16), int(2 ** rng.uniform(0, 14)), int(2 ** rng.uniform(0, 14)))
            for _ in range(500)]:
        q_parts, kv_parts = ctypes.c_int(), ctypes.c_int()
        both = lib().alone(*size, ctypes.byref(q_parts), ctypes.byref(kv_parts))
        _, with_dq, kv = bwd(*size)
        assert not both and q_parts.value == 1 and kv_parts.value == kv      # (the workspace goes by kv_parts)
        split += with_dq > 1
    assert split > 50
