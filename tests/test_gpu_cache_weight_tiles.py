"""Key weights whose first pass goes by tiles of 128 rows: calls with many rows."""
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


def check(ifa, s, lens, W=None):
    want, tol = ref.key_weights(s, lens, W)
    t = ref.on_gpu(s)
    got = ifa.key_weights(t["q8"], t["k8"], t["sq"], t["sk"], W=None if W is None else W.cuda(), lens=None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda"))
    off = (got.cpu().double() - want).abs()
    assert bool((off <= tol).all()), f"off by up to {(off / tol).max().item():.3f} of the tolerance"
    return got


# B, Hkv, G, Nq, Nk, d, lens
WEIGHTS = [
    (3, 88, 2, 32, 70, 64, (70, 3, 0)),                  # half a tile of rows; an empty sequence, one of fewer keys than queries
    (2, 100, 3, 29, 33, 128, (33, 30)),                  # an odd group
    (1, 172, 1, 129, 129, 64, None),                     # prompts; one row in the second tile
    (2, 8, 2, 1500, 400, 64, (400, 399)),                # more queries than keys, many tiles
    (2, 24, 2, 128, 1100, 128, (1100, 700)),             # the keys in parts
    (1, 6, 4, 300, 2000, 64, (1999,)),                   # ... three of them
    (4, 4, 2, 500, 900, 128, (900, 0, 500, 129)),        # padded in front
]


@pytest.mark.parametrize("past", [False, True])
@pytest.mark.parametrize("case", WEIGHTS, ids=[f"{i}" for i in range(len(WEIGHTS))])
def test_key_weights(ifa, case, past):
    B, Hkv, G, Nq, Nk, d, lens = case
    s = ref.problem(52, B, Hkv, G, Nq, Nk, d)
    check(ifa, s, lens, torch.rand(B, Hkv, Nk, generator=torch.Generator().manual_seed(1)) if past else None)


PADDED = (1, 264, 2, 40, 70, 64)


def test_what_padding_queries_hold_does_not_matter(ifa):
    B, Hkv, G, Nq, Nk, d = PADDED
    s = ref.problem(53, B, Hkv, G, Nq, Nk, d)
    for bad in (0.0, math.nan, math.inf):
        s["sq"][:, :, :Nq - 5] = bad
        check(ifa, s, (5,))


def test_what_lies_behind_the_sequence_is_not_looked_at(ifa):
    B, Hkv, G, Nq, Nk, d = PADDED
    s = ref.problem(54, B, Hkv, G, Nq, Nk, d)
    for bad in (math.nan, math.inf):
        s["sk"][:, :, 51:] = bad
        got = check(ifa, s, (51,))
        assert bool((got[:, :, 51:] == 0).all())
