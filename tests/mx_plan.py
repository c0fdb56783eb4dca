"""The plan of the gradients through MXFP4 weights (csrc/tq_mx_plan.hpp), compiled for the host, and the sizes whose plans the tests run."""
from __future__ import annotations

import collections
import ctypes
import functools
import os
import shutil
import subprocess
import tempfile

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_08910_amd", "csrc")
FEW = -1
Plan = collections.namedtuple("Plan", "tile bc bn in_type splits whole stacked")

SRC = """
#include "tq_mx_plan.hpp"
extern "C" void plan(int64_t t, int kb, int n, int mats, int type, int64_t* o) {
  const tq::BwdPlan p = tq::plan_bwd(t, kb, n, mats, type);
  const tq::BwdTile c = p.tile < 0 ? tq::BwdTile{32, 32, {0, 0, 0}, false} : tq::kBwdTiles[p.tile];
  o[0] = p.tile, o[1] = c.bc, o[2] = c.bn, o[3] = c.in_type, o[4] = p.splits, o[5] = p.whole, o[6] = p.stacked;
}
extern "C" int64_t bytes(int n, int type, int64_t t, int mats) { return (int64_t)tq::bwd_bytes(n, type, t, mats); }
extern "C" int64_t pad_of(int n) { return tq::pad_of(n); }
extern "C" int few_waves() { return tq::kFewWaves; }
"""


@functools.lru_cache(None)
def lib():
    cc = shutil.which("g++")
    if cc is None:
        pytest.skip("no host compiler")
    with tempfile.TemporaryDirectory() as d:
        src, out = os.path.join(d, "plan.cpp"), os.path.join(d, "plan.so")
        with open(src, "w") as f:
            f.write(SRC)
        subprocess.run([cc, "-std=c++17", "-O2", "-shared", "-fPIC", "-Wall", "-Werror", "-I", CSRC, src, "-o", out], check=True)
        so = ctypes.CDLL(out)
    i64 = ctypes.c_int64
    so.plan.argtypes, so.plan.restype = [i64, ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.POINTER(i64)], None
    so.bytes.argtypes, so.bytes.restype = [ctypes.c_int, ctypes.c_int, i64, ctypes.c_int], i64
    so.pad_of.restype = i64
    return so


def plan(n, k, t, mats, type_) -> Plan:
    o = (ctypes.c_int64 * 7)()
    lib().plan(t, k // 256, n, mats, type_, o)
    return Plan(*o)


def way(p: Plan):
    """The code that a plan runs: the kernel or tile, how a gradient's parts meet the weights, and who adds them up."""
    tile = "few" if p.tile == FEW else f"{p.bc}x{p.bn}"
    parts = "in type" if p.in_type else "below" if p.stacked else "passes"
    return tile, parts, "last round" if p.whole else "split" if p.splits > 1 else "alone"


# (n, k, t) whose gradients, in every type and by one and two matrices, run through every way above that ordinary sizes take
SIZES = [(66, 11520, 132), (74, 11008, 1411), (224, 1536, 674), (248, 11008, 643), (257, 2816, 279), (318, 11008, 304), (393, 1280, 518),
         (450, 6656, 1153), (493, 3328, 1235), (520, 3328, 257), (605, 5632, 287), (717, 256, 31), (755, 11008, 644), (770, 256, 33),
         (800, 768, 2693), (845, 8448, 68), (846, 768, 324), (964, 256, 1), (972, 11520, 528), (1008, 3328, 1164), (1230, 768, 216),
         (1488, 4352, 130), (1611, 1792, 515), (1627, 512, 172), (1864, 512, 131), (1936, 256, 17), (2002, 768, 71), (2114, 1536, 457),
         (2452, 1280, 394), (2498, 512, 130), (2950, 768, 130)]
