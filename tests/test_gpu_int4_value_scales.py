"""Attention over a cache in 4 bits at the ends of the range of V's scales."""
import pytest
import torch

import int4_reference as ref
import int4_value_scales as exact
from test_gpu_int4 import KINDS, check, ifa, int4, of_kind  # noqa: F401

pytestmark = pytest.mark.gpu


def tiny(turn, shape):
    """Scales below 2^-80, from 2^-118 / 7, which the quantizer still writes, up to just under it; or some of 2^-79 beside them; of either sign in the third."""
    g = torch.Generator().manual_seed(4)
    u = torch.rand(shape, generator=g)
    if turn == "all below":
        return torch.exp2(-100 + 19 * u)
    if turn == "the smallest":
        return torch.where(u < 0.5, 2.0 ** -118 / 7, 2.0 ** -90)
    if turn == "beside larger ones":
        return torch.where(u < 0.5, 2.0 ** -79, 2.0 ** -100)
    if turn == "at the border":
        return torch.where(u < 0.5, 2.0 ** -80 * (1 - 2.0 ** -24), 2.0 ** -80)
    return torch.where(u < 0.1, 0.0, torch.exp2(-100 + 21 * u)) * (torch.randint(0, 2, shape, generator=g) * 2.0 - 1.0)


@pytest.mark.parametrize("turn", ["all below", "the smallest", "beside larger ones", "at the border", "of either sign"])
@pytest.mark.parametrize("kind", KINDS)
def test_scales_below_the_smallest_that_counts(ifa, kind, turn):  # noqa: F811
    """They count as 2^-80 in what weights are rounded to, and as what they are in the output."""
    s, lens = of_kind(kind)
    s["sv"] = tiny(turn, s["sv"].shape).float()
    want, tol = exact.attention(s, lens, tiles=kind.startswith("tiles"))
    assert ((want.abs() > 4 * tol).double().mean() > 0.2) or turn == "the smallest"      # (the tolerance leaves something to see)
    check(int4(ifa, s, None, 0, lens, out_dtype=torch.float32), want, tol)


# B, Hkv, G, Nq, Nk, d, window: tiles of 128 rows
TILES = [(2, 40, 1, 512, 512, 64, None), (2, 40, 2, 300, 700, 128, None), (2, 40, 1, 500, 900, 64, 40), (2, 40, 2, 300, 700, 128, 40), (1, 48, 3, 170, 333, 128, 5)]


@pytest.mark.parametrize("case", TILES, ids=[f"{i}" for i in range(len(TILES))])
def test_hidden_keys_do_not_count(ifa, case):  # noqa: F811
    """Keys with scales 2^39 of the others', some of them later than a query or in front of its window in the same tile of keys: its output is what it is without them."""
    B, Hkv, G, Nq, Nk, d, w = case
    s = ref.problem(9, B, Hkv, G, Nq, Nk, d)
    lens = [Nk, Nk - 37][:B]
    s["sv"] = (s["sv"] * 2.0 ** -20).float()
    if w is None:
        s["sv"][:, :, (Nk - Nq) // 64 * 64 + 63] = 2.0 ** 19             # the last key of the tile in which the queries begin
    else:
        s["sv"][:, :, 31::97] = 2.0 ** 19
    want, tol = exact.attention(s, lens, w, tiles=True)
    assert (want.abs() > 4 * tol).double().mean() > 0.2
    check(int4(ifa, s, w, 0, lens, out_dtype=torch.float32), want, tol)
