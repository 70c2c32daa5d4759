"""The library's own rules for attention over a cache in 4 bits (csrc/intfa_cache_plan.h), compiled for the host."""
import ctypes
import functools
import os
import subprocess
import tempfile

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

_RULES = r"""
#include "intfa_cache_plan.h"
using namespace ifa_cache;
extern "C" void int4(int B, int Hkv, int G, int Nq, int Nk, int d, int window, int sinks, int lens, long *out) {
    const Int4Plan p = int4_plan(B, Hkv, G, Nq, Nk, d, window < Nk ? window : Nk, sinks < Nk ? sinks : Nk, lens);
    out[0] = p.tile, out[1] = p.once, out[2] = p.rows_at_once, out[3] = p.waves, out[4] = p.places, out[5] = p.row_tiles, out[6] = p.parts, out[7] = p.bytes;
}
"""


@functools.lru_cache(maxsize=None)
def rules():
    with tempfile.TemporaryDirectory() as tmp:
        src, lib = os.path.join(tmp, "rules.cpp"), os.path.join(tmp, "rules.so")
        with open(src, "w") as f:
            f.write(_RULES)
        subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_2409_16997_amd", "csrc"), src, "-o", lib], check=True)
        return ctypes.CDLL(lib)


def plan(B, Hkv, G, Nq, Nk, d, window=None, sinks=0, lens=False):
    """How a call is carried out: by tiles of 128 rows or of 16 or 32 (`rows`), in workgroups of 4 or 8 wavefronts (`waves`), each unit's keys whole or in parts (`splits`, or by the lengths: `places`), past
    the caches (`once`); bytes of workspace."""
    out = (ctypes.c_long * 8)()
    rules().int4(B, Hkv, G, Nq, Nk, d, Nk if window is None else window, sinks, int(bool(lens)), out)
    units = B * Hkv
    return {"tile": bool(out[0]), "once": bool(out[1]), "rows": out[2], "waves": out[3], "places": out[4], "row_tiles": out[5], "parts": out[6], "bytes": out[7],
            "splits": 0 if out[4] else out[6] // units, "in_parts": out[6] > units}
