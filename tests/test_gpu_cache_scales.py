"""Scales at the edge of their range in the calls on a quantized cache, on every way through the kernels, against the definitions in 64 bits."""
import math

import pytest
import torch

import cache_reference as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ifa():
    import paper_2409_16997_amd as ifa
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return ifa


def dev_lens(lens):
    return None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")


def window(ifa, s, w, sinks, lens=None, **kw):
    t = ref.on_gpu(s)
    return ifa.int_flash_attn_fwd_window(t["q8"], t["k8"], t["v"], t["sq"], t["sk"], w, sinks, s_V=t["sv"], lens=dev_lens(lens), **kw)


def prefix(ifa, s, lens=None, **kw):
    t = ref.on_gpu(s)
    return ifa.int_flash_attn_fwd_prefix(t["q8"], t["kp8"], t["vp"], t["k8"], t["v"], t["sq"], t["skp"], t["sk"], s_Vp=t["svp"], s_V=t["sv"], lens=dev_lens(lens), **kw)


def check(got, want, tol):
    got = got.cpu().double()
    assert bool(torch.isfinite(got).all()), "not finite"
    off = (got - want).abs()
    assert bool((off <= tol).all()), f"off by up to {(off / tol.clamp_min(1e-300)).max().item():.3f} of the tolerance"


# B, Hkv, G, Nq, Nk, d, window, sinks, lens
WINDOWS = {
    "32 rows": (2, 2, 4, 1, 300, 128, 64, 4, (300, 257)),
    "32 rows, in parts": (1, 1, 8, 2, 5000, 64, 4096, 4, None),
    "tiles": (1, 16, 3, 170, 333, 128, 70, 64, (331,)),
    "tiles, in parts": (1, 8, 4, 140, 2600, 64, 2000, 5, None),
}
# B, Hkv, G, Nq, Np, Nk, d, lens
PREFIXES = {
    "32 rows": (2, 2, 1, 1, 300, 40, 64, (40, 7)),
    "both, 32 rows": (3, 1, 4, 1, 700, 65, 128, (65, 0, 1)),
    "both, tiles": (40, 1, 4, 1, 2000, 200, 64, None),
    "shared tiles, own tiles": (9, 8, 2, 20, 7000, 30, 64, (30, 0, 1, 19, 20, 21, 30, 5, 30)),
    "tiles of both": (3, 8, 2, 100, 70, 100, 128, (100, 99, 1)),
    "tiles of both, in parts": (2, 4, 3, 200, 1000, 300, 64, (300, 0)),
}


@pytest.mark.parametrize("name", WINDOWS)
def test_window_with_values_of_no_scale(ifa, name):
    """s_V = 0 in some heads, and in all: zeros."""
    B, Hkv, G, Nq, Nk, d, w, sinks, lens = WINDOWS[name]
    s = ref.problem(41, B, Hkv, G, Nq, Nk, d, v="int8")
    for zero in (slice(0, None, 2), slice(None)):
        s["sv"][:, zero] = 0.0
        want, tol = ref.attention(s, torch.float32, lens, w, sinks)
        check(window(ifa, s, w, sinks, lens, out_dtype=torch.float32), want, tol)


@pytest.mark.parametrize("which", ["one sequence's", "all own", "shared", "all"])
@pytest.mark.parametrize("name", PREFIXES)
def test_prefix_with_values_of_no_scale(ifa, name, which):
    B, Hkv, G, Nq, Np, Nk, d, lens = PREFIXES[name]
    s = ref.problem(42, B, Hkv, G, Nq, Nk, d, Np=Np, v="int8")
    if which == "one sequence's":
        s["sv"][0] = 0.0
    if which in ("all own", "all"):
        s["sv"][:] = 0.0
    if which in ("shared", "all"):
        s["svp"][:] = 0.0
    want, tol = ref.attention(s, torch.float32, lens)
    check(prefix(ifa, s, lens, out_dtype=torch.float32), want, tol)


@pytest.mark.parametrize("own,shared", [(1e-36, 1.0), (1e-30, 1.0), (1e-12, 100.0), (1.0, 1e-30), (100.0, 1e-12)])
@pytest.mark.parametrize("name", PREFIXES)
def test_prefix_with_scales_far_apart(ifa, name, own, shared):
    """Own and shared V, one of which next to vanishes beside the other.  (Where a scale that is 2^-64 of the other counts as 0, that is 2^-57 of the values beside it: far inside the
    tolerance, which allows 2^-25 of them.)"""
    B, Hkv, G, Nq, Np, Nk, d, lens = PREFIXES[name]
    s = ref.problem(43, B, Hkv, G, Nq, Nk, d, Np=Np, v="int8")
    s["sv"] *= own
    s["svp"] *= shared
    want, tol = ref.attention(s, torch.float32, lens)
    check(prefix(ifa, s, lens, out_dtype=torch.float32), want, tol)


@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("v", ["int8", "fp16"])
@pytest.mark.parametrize("name", list(PREFIXES) + ["tiles, many own parts"])
def test_what_an_empty_sequence_holds_does_not_matter(ifa, name, v, bad):
    """A cache slot of a batch that has no keys yet, behind a prefix: whatever lies in its s_V, V and s_K, its queries get what the shared keys give."""
    B, Hkv, G, Nq, Np, Nk, d, _ = dict(PREFIXES, **{"tiles, many own parts": (3, 1, 2, 600, 4000, 2100, 64, None)})[name]
    lens = [Nk if b % 2 else 0 for b in range(B)]
    s = ref.problem(44, B, Hkv, G, Nq, Nk, d, Np=Np, v=v)
    want, tol = ref.attention(s, torch.float32, lens)
    for b in range(0, B, 2):
        s["sk"][b] = bad
        if v == "int8":
            s["sv"][b] = bad
        else:
            s["v"][b] = bad
    check(prefix(ifa, s, lens, out_dtype=torch.float32), want, tol)


@pytest.mark.parametrize("name", WINDOWS)
def test_what_an_empty_sequence_of_a_window_holds_does_not_matter(ifa, name):
    B, Hkv, G, Nq, Nk, d, w, sinks, _ = WINDOWS[name]
    s = ref.problem(45, B, Hkv, G, Nq, Nk, d, v="int8")
    s["sv"][:], s["sk"][:] = math.nan, math.nan
    got = window(ifa, s, w, sinks, [0] * B, out_dtype=torch.float32)
    assert bool((got == 0).all())


def queries_without_a_scale(s):
    """Every third query row's s_Q 0, the next a subnormal number."""
    flat = s["sq"].view(-1)
    flat[::3] = 0.0
    flat[1::3] = 1e-42
    return s


@pytest.mark.parametrize("name", WINDOWS)
def test_window_with_queries_of_no_scale(ifa, name):
    """s_Q = 0: every score is 0, so all keys that the query sees weigh the same."""
    B, Hkv, G, Nq, Nk, d, w, sinks, lens = WINDOWS[name]
    s = queries_without_a_scale(ref.problem(46, B, Hkv, G, Nq, Nk, d))
    want, tol = ref.attention(s, torch.float32, lens, w, sinks)
    check(window(ifa, s, w, sinks, lens, out_dtype=torch.float32), want, tol)


@pytest.mark.parametrize("name", PREFIXES)
def test_prefix_with_queries_of_no_scale(ifa, name):
    B, Hkv, G, Nq, Np, Nk, d, lens = PREFIXES[name]
    s = queries_without_a_scale(ref.problem(47, B, Hkv, G, Nq, Nk, d, Np=Np))
    want, tol = ref.attention(s, torch.float32, lens)
    check(prefix(ifa, s, lens, out_dtype=torch.float32), want, tol)


# B, Hkv, G, Nq, Nk, d, lens
WEIGHTS = {
    "stored scores": (2, 2, 4, 2, 700, 64, (700, 1)),
    "32 rows": (1, 2, 3, 40, 300, 128, (299,)),
    "tiles": (3, 88, 2, 32, 70, 64, (70, 3, 40)),
    "tiles, in parts": (2, 24, 2, 128, 1100, 128, (1100, 700)),
}


@pytest.mark.parametrize("name", WEIGHTS)
def test_key_weights_with_queries_of_no_scale(ifa, name):
    B, Hkv, G, Nq, Nk, d, lens = WEIGHTS[name]
    s = queries_without_a_scale(ref.problem(48, B, Hkv, G, Nq, Nk, d))
    want, tol = ref.key_weights(s, lens)
    t = ref.on_gpu(s)
    check(ifa.key_weights(t["q8"], t["k8"], t["sq"], t["sk"], lens=dev_lens(lens)), want, tol)


@pytest.mark.parametrize("name", WEIGHTS)
def test_keys_of_no_scale(ifa, name):
    """s_K = 0: such keys score 0 with every query."""
    B, Hkv, G, Nq, Nk, d, lens = WEIGHTS[name]
    s = ref.problem(49, B, Hkv, G, Nq, Nk, d)
    s["sk"].view(-1)[::3] = 0.0
    want, tol = ref.key_weights(s, lens)
    t = ref.on_gpu(s)
    check(ifa.key_weights(t["q8"], t["k8"], t["sq"], t["sk"], lens=dev_lens(lens)), want, tol)
    want, tol = ref.attention(s, torch.float32, lens, 100, 3)
    check(window(ifa, s, 100, 3, lens, out_dtype=torch.float32), want, tol)
