"""The cases of test_gpu_int4_large.py reach every kernel that reads past the caches, by the library's own rules, and each such kernel is one of few rows in four wavefronts."""
import itertools

import int4_routes as routes
import test_gpu_int4_large as tests


def test_every_kernel_past_the_caches():
    seen = set()
    for B, Hkv, G, Nq, Nk, d, w, sinks, lens in tests.CASES:
        p = routes.plan(B, Hkv, G, Nq, Nk, d, w, sinks, lens is not None)
        assert p["once"], (B, Hkv, G, Nq, Nk, d)
        seen.add((d, p["rows"], "by lengths" if p["places"] else "in parts" if p["in_parts"] else "whole"))
    assert seen == set(itertools.product((64, 128), (16, 32), ("whole", "in parts", "by lengths")))


def test_no_other_kernel_reads_past_them():
    for units, rows, Nk, d in itertools.product((1, 8, 64, 128, 512, 4096), (1, 16, 17, 32, 33, 128, 1000), (64, 700, 896, 1024, 4000, 100000), (64, 128)):
        p = routes.plan(1, units, rows, 1, Nk, d)
        assert not p["once"] or (not p["tile"] and p["waves"] == 4 and p["row_tiles"] == 1)
