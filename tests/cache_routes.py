"""The library's own rules for the calls on a quantized cache (csrc/intfa_cache_plan.h), compiled for the host: tests say which kernels they reach without a line of their own."""
import ctypes
import functools
import os
import subprocess
import tempfile

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

_RULES = r"""
#include "intfa_cache_plan.h"
using namespace ifa_cache;
extern "C" void attention(int B, int Hkv, int G, int Nq, int Np, int Nk, int window, int sinks, int key_bytes, int *out) {
    const AttentionPlan p = attention_plan(B, Hkv, G, Nq, Np, Nk, window < Nk ? window : Nk, sinks < Nk ? sinks : Nk, key_bytes);
    out[0] = p.way, out[1] = p.shared, out[2] = p.own, out[3] = p.ahead, out[4] = p.once, out[5] = p.join();
}
extern "C" void weights(int B, int Hkv, int G, int Nq, int Nk, int d, int *out) {
    const WeightsPlan p = weights_plan(B, Hkv, G, Nq, Nk, d);
    out[0] = p.few, out[1] = p.stored, out[2] = p.once, out[3] = p.parts, out[4] = p.slices;
}
extern "C" int rounds(int Nk) { return evict_rounds(Nk); }
"""
WAYS = ("few", "both few", "both tile", "tile", "tile front", "tile apart")


@functools.lru_cache(maxsize=None)
def rules():
    with tempfile.TemporaryDirectory() as tmp:
        src, lib = os.path.join(tmp, "rules.cpp"), os.path.join(tmp, "rules.so")
        with open(src, "w") as f:
            f.write(_RULES)
        subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_2409_16997_amd", "csrc"), src, "-o", lib], check=True)
        return ctypes.CDLL(lib)


def attention(B, Hkv, G, Nq, Nk, d, window=None, sinks=0, Np=0, v="fp16"):
    """How an attention call is carried out: `way` ("few": the 32-row kernel; "both few", "both tile": shared and own keys in one launch; "tile": tiles of 128 rows on own keys, "tile
    front" on shared and then own ones, "tile apart" on each), parts of the shared and of the own keys, and for "few" the tiles copied ahead and whether K and V go past the caches."""
    out = (ctypes.c_int * 6)()
    rules().attention(B, Hkv, G, Nq, Np, Nk, Nk if window is None else window, sinks, (3 if v == "fp16" else 2) * d, out)
    return {"way": WAYS[out[0]], "shared": out[1], "own": out[2], "ahead": out[3], "once": bool(out[4]), "join": bool(out[5])}


def weights(B, Hkv, G, Nq, Nk, d):
    """How key weights are found: first pass by 32 rows (`few`) or tiles of 128, scores `stored` or computed again, K past the caches (`once`), parts of the keys, slices of the rows."""
    out = (ctypes.c_int * 5)()
    rules().weights(B, Hkv, G, Nq, Nk, d, out)
    return {"few": bool(out[0]), "stored": bool(out[1]), "once": bool(out[2]), "parts": out[3], "slices": out[4]}


def evict_rounds(Nk):
    """How many rounds of 4096 keys have their weights in registers (0: read again)."""
    return rules().rounds(Nk)
