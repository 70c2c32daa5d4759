"""Attention over a quantized cache where one key outweighs a long flat rest by 12 to 18 nats: what the rest adds up to, against the closed form in 64 bits.

The first key has S = T and the value 0, all others S = 0 and values between 1 and 2: O = e^-T sum v / (1 + n e^-T), all of it from weights of 2^-17 to 2^-26 of the largest.
How far a kernel may be off:
  weights   a weight is rounded by 2^-11 of itself, or by `cut` of the largest of its row where that is more: the fp16 half step of its lowest binades, 2^-25, over the fp16 weight of the
            largest key, which is 2^15 in the kernel for 32 rows and at least 2^7 in tiles.  Numerator and denominator, each relatively.
  scores    8 T 2^-24 absolutely, and exp2 by 2^-22 (as in cache_reference)
  sums      O by n / 16 additions (16 keys to an instruction) of 2^-24 each, all in one direction at worst; l, beside whose largest summand the rest is small, by n / 16 additions of
            2^-24 of l, too (a lane has 16 of 32 keys or more to an addition)
  output    fp32: 2^-24
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ifa():
    import paper_2409_16997_amd as ifa
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return ifa


def problem(T, heads, Nq, Nk, d, v, seed=0):
    """One head's operands, for `heads` heads (the kernels see copies); and e^-T as the stored scales have it."""
    g = torch.Generator().manual_seed(seed)
    q8 = torch.full((1, 1, Nq, d), 64, dtype=torch.int8)
    k8 = torch.zeros((1, 1, Nk, d), dtype=torch.int8)
    k8[:, :, 0] = 64
    sq = torch.full((1, 1, Nq), T / (4096.0 * d))
    sk = torch.ones(1, 1, Nk)
    if v == "int8":
        v8, sv = torch.randint(64, 128, (1, 1, Nk, d), generator=g).to(torch.int8), torch.full((1, 1), 1.0 / 64)
    else:
        v8, sv = (torch.rand((1, 1, Nk, d), generator=g) + 1.0).half(), None
    v8[:, :, 0] = 0
    many = [None if x is None else x.cuda().expand(1, heads, *x.shape[2:]).contiguous() for x in (q8, k8, v8, sq, sk, sv)]
    values = v8[0, 0].double() * (1.0 if sv is None else 1.0 / 64)
    return many, values, math.exp(-sq[0, 0, 0].double().item() * 4096 * d)


def expected(values, small, Nq, cut, T):
    """(O [Nq, d], tolerance); query i sees the first Nk - Nq + 1 + i keys."""
    n = values.shape[0]
    total = values.cumsum(0)[n - Nq:]
    count = torch.arange(n - Nq, n).double()[:, None]            # keys beside the first
    O = small * total / (1 + small * count)
    rel = 2 * (2.0 ** -11 + cut / small + 8 * T * 2.0 ** -24 + 2.0 ** -22) + 2 * n / 16 * 2.0 ** -24 + 2.0 ** -24
    return O, rel * O


FEW, TILE = 2.0 ** -25 / 2 ** 15, 2.0 ** -25 / 2 ** 7
# heads, Nq, Nk, d, the smallest weight's rounding
CASES = {
    "32 rows": (130, 1, 16384, 64, FEW),
    "32 rows, in parts": (2, 3, 40000, 128, FEW),
    "tiles": (260, 33, 9000, 64, TILE),
    "tiles, in parts": (65, 40, 16000, 128, TILE),
}


@pytest.mark.parametrize("T", [12.0, 14.0, 16.0, 18.0])
@pytest.mark.parametrize("v", ["fp16", "int8"])
@pytest.mark.parametrize("name", CASES)
def test_a_long_flat_rest(ifa, name, v, T):
    heads, Nq, Nk, d, cut = CASES[name]
    (q, k, v8, sq, sk, sv), values, small = problem(T, heads, Nq, Nk, d, v)
    O, tol = expected(values, small, Nq, cut, T)
    got = ifa.int_flash_attn_fwd_window(q, k, v8, sq, sk, Nk, s_V=sv, out_dtype=torch.float32)[0].cpu()
    assert bool((got == got[:1]).all())
    off = (got[0].double() - O).abs()
    assert bool((off <= tol).all()), f"off by up to {(off / O).max().item():.2e} of O, {(off / tol).max().item():.3f} of the tolerance"


# heads, sequences, Nq, Np, Nk, d: the first key is the first shared one
PREFIXES = {
    "32 rows": (2, 2, 1, 300, 150, 64, FEW),
    "both, 32 rows": (2, 3, 1, 20000, 3000, 64, FEW),
    "both, tiles": (1, 40, 1, 12000, 2000, 128, TILE),
    "tiles of both": (60, 3, 128, 6000, 500, 64, TILE),
    "shared tiles, own tiles": (8, 10, 40, 30000, 300, 64, TILE),
}


@pytest.mark.parametrize("T", [12.0, 16.0, 18.0])
@pytest.mark.parametrize("v", ["fp16", "int8"])
@pytest.mark.parametrize("name", PREFIXES)
def test_a_long_flat_rest_behind_a_prefix(ifa, name, v, T):
    heads, B, Nq, Np, Nk, d, cut = PREFIXES[name]
    (q, k, v8, sq, sk, sv), values, small = problem(T, heads, Nq, Np + Nk, d, v)
    O, tol = expected(values, small, Nq, cut, T)

    def batch(x):
        return x.expand(B, *x.shape[1:]).contiguous()

    own = [batch(x[:, :, Np:]) for x in (k, v8, sk)]
    got = ifa.int_flash_attn_fwd_prefix(batch(q), k[0, :, :Np].contiguous(), v8[0, :, :Np].contiguous(), own[0], own[1], batch(sq), sk[0, :, :Np].contiguous(), own[2],
                                        s_Vp=None if sv is None else sv[0], s_V=None if sv is None else batch(sv), out_dtype=torch.float32).cpu()
    assert bool((got == got[:1, :1]).all())
    off = (got[0, 0].double() - O).abs()
    assert bool((off <= tol).all()), f"off by up to {(off / O).max().item():.2e} of O, {(off / tol).max().item():.3f} of the tolerance"
