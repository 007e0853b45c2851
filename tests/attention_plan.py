"""Which kernels the attention operators take, asked on the host: csrc/jet_attn_plan.h compiled with g++, no GPU involved."""
from __future__ import annotations

import ctypes
import os
import subprocess
import tempfile

from launch_plan import CSRC

SHIM = """
#include "jet_attn_plan.h"
extern "C" int few_rows(long n, long Tq, long Tk, long group, long n_kv, int dim) { return jet::few_row_tiles(n, Tq, Tk, group, n_kv, dim); }
extern "C" int split(long n, long Tq, long Tk, long group, long n_kv, int dim, int causal, int* out) {
    const jet::Split s = jet::dkdv_split(n, Tq, Tk, group, n_kv, dim, causal);
    out[0] = s.parts; out[1] = s.rows;
    return s.few;
}
extern "C" int chunk(long B, long n_q, long n_kv, int dim, int fp8, long capacity) {
    return jet::decode_chunk(B * n_kv * ((n_q / n_kv + 15) / 16), capacity, jet::decode_waves(dim, fp8));
}
extern "C" int qk_few(long T, long n_q, long n_kv, int dim, int cached) { return jet::qk_few_heads(T, n_q, n_kv, dim, cached); }
extern "C" int qk_bwd_few(long T, long n_q, long n_kv, int dim) { return jet::qk_bwd_groups(T, n_q, n_kv, dim).few; }
"""
_lib = None


def lib():
    global _lib
    if _lib is None:
        with tempfile.TemporaryDirectory() as d:
            src, so = os.path.join(d, "plan.cpp"), os.path.join(d, "plan.so")
            with open(src, "w") as f:
                f.write(SHIM)
            subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", f"-I{CSRC}", src, "-o", so], check=True)
            _lib = ctypes.CDLL(so)
        i, l = ctypes.c_int, ctypes.c_long
        _lib.few_rows.argtypes = [l] * 5 + [i]
        _lib.split.argtypes = [l] * 5 + [i, i, ctypes.POINTER(i)]
        _lib.chunk.argtypes = [l] * 3 + [i, i, l]
        _lib.qk_few.argtypes = [l] * 3 + [i, i]
        _lib.qk_bwd_few.argtypes = [l] * 3 + [i]
    return _lib


def _sizes(case):
    lq, prefix, n_q, n_kv, dim, _ = case
    return len(lq), sum(lq), sum(lq) + prefix * len(lq), n_q // n_kv, n_kv, dim


def rows(case) -> str:
    """The kernel of the forward pass and of dq: tiles of 128 rows ('many') or of 32 ('few')."""
    return "few" if lib().few_rows(*_sizes(case)) else "many"


def keys(case):
    """The kernel of dk and dv, and how many workgroups have the rows of the first tile of each sequence."""
    out = (ctypes.c_int * 2)()
    few = lib().split(*_sizes(case), case[5], out)
    parts, each = out
    group = case[2] // case[3]
    return "few" if few else "many", [max(1, min(parts, -(-n * group // each))) for n in case[0]]


def chunks(B, n_q, n_kv, dim, fp8, capacity) -> int:
    return -(-capacity // lib().chunk(B, n_q, n_kv, dim, fp8, capacity))


def heads(T, n_q, n_kv, dim, cached=False) -> int:
    return 1 if lib().qk_few(T, n_q, n_kv, dim, cached) else 4


def heads_bwd(T, n_q, n_kv, dim) -> int:
    return 1 if lib().qk_bwd_few(T, n_q, n_kv, dim) else 4
