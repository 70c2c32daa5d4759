"""Attention over more than 64 MB of a cache in 4 bits, which is read past the caches: the kernels that only such calls reach, against the definition in 64 bits."""
import pytest
import torch

import int4_reference as ref
from test_gpu_int4 import check, ifa, int4  # noqa: F401

pytestmark = pytest.mark.gpu

# B, Hkv, G, Nq, Nk, d, window, sinks, lens
CASES = [
    (64, 8, 2, 1, 1000, 128, None, 0, None),             # whole, 16 rows
    (61, 9, 2, 1, 963, 128, None, 0, tuple(963 - 15 * b for b in range(61))),
    (64, 8, 5, 4, 1000, 128, None, 0, None),             # ... 32 rows
    (1, 8, 4, 1, 63001, 128, None, 0, None),             # in parts
    (2, 4, 6, 4, 63000, 128, None, 0, None),
    (2, 4, 2, 2, 70000, 128, 62000, 100, (69999, 65001)),
    (16, 4, 2, 1, 8000, 128, None, 0, tuple(8000 - 31 * b for b in range(16))),       # by the lengths
    (16, 4, 20, 1, 8100, 128, None, 0, (8100, 0, 1, 64) + tuple(600 * b + 5 for b in range(12))),
    (64, 8, 2, 1, 1900, 64, None, 0, None),
    (64, 8, 5, 4, 1850, 64, None, 0, tuple(1850 - 3 * b for b in range(64))),
    (1, 8, 4, 1, 120001, 64, None, 0, None),
    (2, 4, 6, 4, 118000, 64, None, 0, None),
    (16, 4, 2, 1, 15000, 64, None, 0, tuple(15000 - 400 * b for b in range(16))),
    (16, 4, 20, 1, 15000, 64, 14900, 64, (15000, 0, 1) + tuple(1000 * b + 63 for b in range(13))),
]


@pytest.mark.parametrize("case", CASES, ids=[f"{i}" for i in range(len(CASES))])
def test_read_past_the_caches(ifa, case):  # noqa: F811
    B, Hkv, G, Nq, Nk, d, w, sinks, lens = case
    s = ref.problem(13, B, Hkv, G, Nq, Nk, d)
    want, tol = ref.attention(s, torch.float16, lens, w, sinks)
    check(int4(ifa, s, w, sinks, lens), want, tol)
