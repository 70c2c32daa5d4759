"""Which kernels the GPU tests of the calls on a quantized cache reach, by the library's own rules."""
import pytest

import cache_routes
import test_gpu_cache_attention as attention_tests
import test_gpu_cache_far_weights as far_tests
import test_gpu_cache_scales as scale_tests
import test_gpu_cache_weight_tiles as tile_tests
import test_gpu_cache_weights as weights_tests


def window(case, v="fp16"):
    B, Hkv, G, Nq, Nk, d, w, sinks = case[:8]
    return cache_routes.attention(B, Hkv, G, Nq, Nk, d, w, sinks, v=v)


def prefix(case, v="fp16"):
    B, Hkv, G, Nq, Np, Nk, d = case[:7]
    return cache_routes.attention(B, Hkv, G, Nq, Nk, d, Np=Np, v=v)


def weights(case):
    return cache_routes.weights(*case[:6])


def test_the_windows_reach_every_kernel_of_own_keys():
    seen = {(p["way"], p["own"] > 1) for p in map(window, attention_tests.WINDOWS)}
    assert seen == {(way, parts) for way in ("few", "tile") for parts in (False, True)}
    assert {p["ahead"] for p in map(window, attention_tests.WINDOWS) if p["way"] == "few"} == {2}          # (one tile ahead, and past the caches: the large calls, by themselves)


def test_the_prefixes_reach_every_kernel():
    plans = [prefix(c) for c in attention_tests.PREFIXES]
    assert {p["way"] for p in plans} == {"few", "both few", "both tile", "tile front", "tile apart"}
    assert {p["own"] > 1 for p in plans if p["way"] == "tile front"} == {False, True}
    assert {p["shared"] + p["own"] > 8 for p in plans if p["join"]} == {False, True}                      # both forms of the join


def test_the_padding_and_hidden_keys_reach_both_kernels():
    assert [cache_routes.attention(2, Hkv, 2, Nq, 260, 64, 40, 2)["way"] for Hkv, Nq in ((1, 9), (16, 200))] == ["few", "tile"]
    assert cache_routes.attention(1, 16, 2, 160, 900, 64, 100, 70)["way"] == "tile"


def test_the_key_weights_reach_every_kernel():
    plans = [weights(c) for c in weights_tests.WEIGHTS + tile_tests.WEIGHTS]
    assert {(p["few"], p["stored"], p["parts"] > 1) for p in plans} == {(True, True, False), (True, True, True), (True, False, False), (True, False, True), (False, False, False), (False, False, True)}
    assert {p["slices"] > 1 for p in plans if not p["stored"]} == {False, True}
    assert not any(weights(c)["few"] for c in tile_tests.WEIGHTS)
    of_padding = [cache_routes.weights(1, Hkv, G, Nq, 260, 64) for Hkv, G, Nq in ((1, 1, 9), (1, 2, 30))] + [cache_routes.weights(*tile_tests.PADDED)]
    assert [(p["few"], p["stored"]) for p in of_padding] == [(True, True), (True, False), (False, False)]


def test_where_scores_are_stored():
    for d, most in ((64, 12), (128, 16)):
        assert [cache_routes.weights(4, 8, rows, 1, 8192, d)["stored"] for rows in (1, most, most + 1)] == [True, True, False]


# First passes on the faster side of the line between 32 rows and tiles of 128, where the other one takes at least 5 % longer
@pytest.mark.parametrize("heads,rows,Nk,d,few", [
    (8, 400, 1024, 128, True), (32, 128, 1024, 128, True), (16, 512, 1024, 128, True), (128, 64, 512, 128, True), (8, 200, 4096, 128, True), (128, 128, 256, 64, True), (4, 100, 8192, 64, True),
    (8, 200, 8192, 128, False), (16, 256, 4096, 128, False), (128, 128, 2048, 128, False), (16, 100, 16384, 128, False), (256, 200, 256, 128, False), (8, 384, 16384, 64, False),
    (32, 512, 2048, 64, False), (256, 512, 2048, 64, False)])
def test_first_passes_on_the_faster_side(heads, rows, Nk, d, few):
    assert cache_routes.weights(1, heads, 1, rows, Nk, d)["few"] == few


def test_the_evictions_reach_every_form():
    assert {cache_routes.evict_rounds(c[2]) for c in weights_tests.EVICTIONS} == {0, 1, 4, 8}


def test_the_names_of_the_scale_cases():
    assert {n: (window(c)["way"], window(c)["own"] > 1) for n, c in scale_tests.WINDOWS.items()} == {
        "32 rows": ("few", False), "32 rows, in parts": ("few", True), "tiles": ("tile", False), "tiles, in parts": ("tile", True)}
    of = {n: prefix(c, "int8") for n, c in scale_tests.PREFIXES.items()}
    assert {n: p["way"] for n, p in of.items()} == {"32 rows": "few", "both, 32 rows": "both few", "both, tiles": "both tile", "shared tiles, own tiles": "tile apart",
                                                    "tiles of both": "tile front", "tiles of both, in parts": "tile front"}
    assert of["tiles of both"]["own"] == 1
    # 16 blocks of shared keys in 5 parts of 4: the last has no block of a sequence without keys
    assert of["tiles of both, in parts"]["own"] == 5
    of = {n: weights(c) for n, c in scale_tests.WEIGHTS.items()}
    assert {n: (p["few"], p["stored"], p["parts"] > 1) for n, p in of.items()} == {
        "stored scores": (True, True, True), "32 rows": (True, False, False), "tiles": (False, False, False), "tiles, in parts": (False, False, True)}


def test_the_names_of_the_cases_of_far_weights():
    of = {n: cache_routes.attention(1, heads, 1, Nq, Nk, d) for n, (heads, Nq, Nk, d, _) in far_tests.CASES.items()}
    assert {n: (p["way"], p["own"] > 1) for n, p in of.items()} == {
        "32 rows": ("few", False), "32 rows, in parts": ("few", True), "tiles": ("tile", False), "tiles, in parts": ("tile", True)}
    of = {n: cache_routes.attention(B, heads, 1, Nq, Nk, d, Np=Np) for n, (heads, B, Nq, Np, Nk, d, _) in far_tests.PREFIXES.items()}
    assert {n: p["way"] for n, p in of.items()} == {"32 rows": "few", "both, 32 rows": "both few", "both, tiles": "both tile", "tiles of both": "tile front", "shared tiles, own tiles": "tile apart"}
