"""Which kernels the GPU tests of the 4-bit cache reach, by the library's own rules, and that a workspace for a shape fits the call with lengths and without."""
import random

import pytest

import int4_routes as routes
import test_gpu_int4 as tests


def of(case):
    B, Hkv, G, Nq, Nk, d, w, sinks, lens = case
    return routes.plan(B, Hkv, G, Nq, Nk, d, w, sinks, lens is not None)


def kind(p):
    if p["tile"]:
        return "tiles", p["in_parts"]
    return p["rows"], p["waves"], "by lengths" if p["places"] else "in parts" if p["in_parts"] else "whole"


def test_the_cases_reach_every_kernel():
    for d in (64, 128):
        seen = {kind(of(c)) for c in tests.CASES + tests.LONG + tests.UNEVEN if c[5] == d}
        assert seen >= {("tiles", False), (16, 4, "whole"), (32, 4, "whole"), (16, 8, "whole"), (32, 8, "whole"), (16, 4, "in parts"), (32, 4, "in parts")}, (d, seen)
    assert {kind(of(c)) for c in tests.UNEVEN} == {(16, 4, "by lengths"), (32, 4, "by lengths")}
    assert any(kind(of(c)) == ("tiles", True) for c in tests.CASES + tests.LONG)
    assert any(of(c)["row_tiles"] > 1 and of(c)["places"] for c in tests.UNEVEN)
    splits = {of(c)["splits"] > 8 for c in tests.CASES + tests.LONG if of(c)["splits"] > 1}
    assert splits == {False, True}                       # both forms of the join


def test_the_names_of_the_kinds():
    of_kind = {n: kind(routes.plan(*c, lens=True)) for n, c in tests.KINDS.items()}
    assert of_kind == {"whole": (16, 4, "whole"), "eight wavefronts": (16, 8, "whole"), "in parts": (16, 4, "in parts"), "by lengths": (16, 4, "by lengths"), "32 rows": (32, 4, "whole"),
                       "tiles": ("tiles", False), "tiles in parts": ("tiles", True)}


def test_the_workspace_of_a_shape_serves_it_with_lengths_and_without():
    rng = random.Random(1)
    for _ in range(20000):
        B, Hkv, G = rng.choice([1, 2, 3, 8, 16, 64, 300]), rng.choice([1, 2, 4, 8, 32]), rng.choice([1, 2, 4, 7, 8])
        Nq, Nk = rng.choice([1, 2, 5, 16, 40, 128, 500, 4000]), rng.choice([1, 64, 300, 700, 1000, 3000, 9000, 40000, 200000])
        d, w = rng.choice([64, 128]), rng.choice([None, 1, 100, 1000, 5000])
        with_lens, without = (routes.plan(B, Hkv, G, Nq, Nk, d, w, 4, lens) for lens in (True, False))
        assert with_lens["bytes"] >= without["bytes"], (B, Hkv, G, Nq, Nk, d, w)
        assert with_lens["places"] == 0 or with_lens["parts"] == B * Hkv + with_lens["places"]


def test_how_many_parts():
    """Up to 64 a unit, 128 where there are one or two groups of rows; a case of the GPU tests has more than 64."""
    assert [routes.plan(1, u, 1, 1, 200000, 128)["splits"] for u in (1, 2, 3, 8, 32)] == [128, 128, 64, 64, 16]
    assert max(of(c)["splits"] for c in tests.LONG) > 64


@pytest.mark.parametrize("units,rows,Nk,d,want", [
    (8, 4, 300, 128, (16, 4, "whole")), (8, 4, 700, 128, (16, 8, "whole")), (8, 4, 2200, 128, (16, 4, "in parts")), (64, 4, 1100, 128, (16, 4, "in parts")), (128, 4, 1500, 128, (16, 4, "whole")),
    (256, 4, 3000, 128, (16, 4, "whole")), (8, 4, 700, 64, (16, 8, "whole")), (64, 40, 16000, 128, (32, 4, "in parts")), (64, 100, 1000, 128, (32, 4, "whole")), (64, 100, 16000, 128, ("tiles", True)),
    (16, 256, 4000, 128, (32, 4, "in parts")), (8, 4096, 4096, 128, ("tiles", True)), (16, 4096, 4096, 128, ("tiles", False)),
    (192, 100, 300, 128, ("tiles", False)), (128, 100, 300, 128, (32, 4, "whole")), (128, 256, 456, 64, ("tiles", False)),
    (160, 100, 300, 128, ("tiles", False)), (80, 256, 456, 128, ("tiles", False)), (64, 256, 456, 128, (32, 4, "whole")), (64, 256, 1000, 64, (32, 4, "whole")),
    (400, 40, 300, 128, ("tiles", False)), (600, 80, 500, 64, ("tiles", False)), (300, 96, 2000, 128, (32, 4, "whole")), (600, 32, 64, 128, ("tiles", False)), (600, 32, 300, 128, (32, 4, "whole")),
    (600, 16, 64, 128, (16, 4, "whole"))])
def test_on_the_faster_side(units, rows, Nk, d, want):
    assert kind(routes.plan(1, units, rows, 1, Nk, d)) == want
