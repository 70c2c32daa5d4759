"""Which kernels test_gpu_int4_value_scales.py reaches, by the library's own rules."""
import int4_routes as routes
import test_gpu_int4_value_scales as tests


def test_hidden_keys_in_tiles_of_both_sizes():
    plans = [(routes.plan(B, Hkv, G, Nq, Nk, d, w, 0, True), d, w) for B, Hkv, G, Nq, Nk, d, w in tests.TILES]
    assert all(p["tile"] for p, _, _ in plans)
    assert {(d, w is None) for _, d, w in plans} == {(64, True), (64, False), (128, True), (128, False)}
