"""Which kernels the embedding, layer norm and clipping operators take, asked on the host: csrc/jet_step_plan.h compiled with g++, no GPU."""
from __future__ import annotations

import ctypes
import os
import subprocess
import tempfile

from launch_plan import CSRC

SHIM = """
#include "jet_step_plan.h"
using namespace jet;
extern "C" long number(int i) {
    const long v[] = {kSortBlock, kNarrowRows, kEmbedDirect, kPlaceTokens, kLongRun, kClipBatch, kClipChunk, kClipGroups, kClipFuse, kClipInPlace, kClipKeep,
                      kRankTokens, kRankBlocks, kMergeRuns};
    return v[i];
}
extern "C" int block(long T, long H) { return embed_block(T, H); }
extern "C" long later(long bytes) { return embed_zeros_later(bytes); }
extern "C" int by_runs(long T, long H) { return embed_by_runs(T, H); }
extern "C" int merges(long T) { return embed_merges(T); }
extern "C" long space(long T, long H, int what) { const EmbedSpace s = embed_space(T, H); return what == 0 ? s.tmp : what == 1 ? s.partial : s.bytes; }
extern "C" int nt(long bytes) { return writes_past_the_caches(bytes); }
extern "C" int team(long M, long K, int both) { const NormTeam t = norm_team(M, K, both); return t.waves * 100 + t.pieces; }
extern "C" int bwd_team(long K) { const NormTeam t = norm_bwd_team(K); return t.waves * 100 + t.pieces; }
extern "C" int norm_alone(long bytes, long sums) { return clip_norm_alone(bytes, sums); }
extern "C" long clip_sums(long chunks) { return clip_groups(chunks); }
extern "C" long bwd_groups(long M, long K) { return norm_bwd_groups(M, K); }
"""
NAMES = ["sort_block", "narrow_rows", "direct", "places", "long_run", "batch", "chunk", "groups", "fuse", "in_place", "keep", "rank_tokens", "rank_blocks", "merge_runs"]
_lib = None


def lib():
    global _lib
    if _lib is None:
        with tempfile.TemporaryDirectory() as d:
            src, so = os.path.join(d, "plan.cpp"), os.path.join(d, "plan.so")
            with open(src, "w") as f:
                f.write(SHIM)
            subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-Wno-unused-variable", "-shared", "-fPIC", f"-I{CSRC}", src, "-o", so], check=True)
            _lib = ctypes.CDLL(so)
        i, l = ctypes.c_int, ctypes.c_long
        for name, res, args in (("number", l, [i]), ("block", i, [l, l]), ("merges", i, [l]), ("by_runs", i, [l, l]), ("later", l, [l]), ("space", l, [l, l, i]), ("nt", i, [l]), ("team", i, [l, l, i]), ("bwd_team", i, [l]),
                                ("bwd_groups", l, [l, l]), ("norm_alone", i, [l, l]), ("clip_sums", l, [l])):
            f = getattr(_lib, name)
            f.restype, f.argtypes = res, args
    return _lib


def numbers():
    return {name: lib().number(i) for i, name in enumerate(NAMES)}


def order(T):
    """How the order of T tokens is found."""
    n = numbers()
    return "direct" if T <= n["direct"] else "places" if T <= n["places"] else "sort"


def team(M, K, both=False):
    return divmod(lib().team(M, K, both), 100)


def bwd_team(K):
    return divmod(lib().bwd_team(K), 100)
