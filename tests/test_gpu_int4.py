"""Attention over a cache held in 4 bits against its definition in 64 bits."""
import math

import pytest
import torch

import int4_reference as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ifa():
    import paper_2409_16997_amd as ifa
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return ifa


def dev_lens(lens):
    return None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")


def int4(ifa, s, window=None, sinks=0, lens=None, **kw):
    t = ref.on_gpu(s)
    return ifa.int_flash_attn_fwd_int4(t["q8"], t["k4"], t["v4"], t["sq"], t["sk"], t["sv"], window=window, sinks=sinks, lens=dev_lens(lens), **kw)


def check(got, want, tol):
    got = got.cpu().double()
    assert bool(torch.isfinite(got).all())
    off = (got - want).abs()
    worst = (off / tol.clamp_min(1e-300)).max().item()
    assert worst <= 1.0, f"off by up to {worst:.3f} of the tolerance"


# B, Hkv, G, Nq, Nk, d, window, sinks, lens
CASES = [
    (1, 1, 1, 1, 1, 64, None, 0, None),                  # one key
    (1, 1, 1, 1, 1, 128, None, 0, None),
    (2, 3, 1, 1, 33, 128, None, 0, None),
    (2, 3, 1, 1, 64, 64, None, 0, None),                 # a tile, and one key more
    (2, 3, 1, 1, 65, 128, None, 0, None),
    (2, 2, 4, 1, 300, 128, None, 0, (300, 257)),         # a decode step, grouped heads
    (2, 2, 4, 1, 300, 64, 64, 4, (300, 257)),
    (1, 1, 8, 1, 5000, 128, None, 0, None),              # shared out over workgroups
    (1, 2, 16, 1, 9000, 64, None, 0, (8999,)),
    (3, 2, 2, 1, 2500, 64, 2000, 100, (2500, 0, 1)),     # an empty sequence, one of one key
    (1, 2, 3, 5, 700, 128, 100, 7, (650,)),              # draft tokens, an odd group
    (2, 2, 8, 4, 3000, 128, None, 0, (2999, 3)),         # 32 rows; more queries than keys
    (1, 1, 7, 9, 1200, 64, 1000, 64, (1199,)),
    (2, 2, 8, 5, 1500, 128, None, 0, (1500, 700)),       # 40 rows
    (2, 1, 1, 40, 40, 128, 3, 2, (40, 17)),              # a prompt, padded in front
    (1, 2, 1, 129, 129, 64, 1, 0, None),                 # every query sees itself alone
    (1, 1, 2, 130, 257, 128, 64, 64, None),              # a chunk; sinks as many as the window
    (1, 1, 4, 200, 200, 64, 500, 3, None),               # a window beyond the sequence
    (2, 1, 1, 31, 95, 128, 32, 300, (95, 20)),           # more sinks than keys
    (1, 3, 1, 300, 300, 128, 129, 1, (290,)),
    (4, 1, 1, 2, 4, 64, 2, 1, (4, 3, 2, 1)),
    (2, 8, 2, 200, 500, 64, 64, 100, (500, 333)),        # tiles of 128 rows: the seam between sinks and window inside a block, ...
    (1, 16, 3, 170, 333, 128, 70, 64, (331,)),           # ... at its end
    (3, 4, 4, 130, 130, 128, None, 0, (130, 0, 77)),     # padded in front
    (1, 12, 1, 400, 650, 64, None, 0, None),
    (2, 6, 4, 129, 700, 128, 10 ** 6, 0, (700, 650)),
    (1, 8, 4, 300, 1300, 128, None, 0, (1290,)),         # a chunk deep in its sequence
    (9, 1, 5, 3, 64, 64, 7, 1, (64, 0, 1, 2, 3, 4, 31, 32, 33)),
    (1, 9, 1, 513, 513, 64, None, 0, (700,)),            # a length beyond the buffer
    (2, 8, 2, 128, 1000, 128, 1, 1, (1000, -5)),
]


@pytest.mark.parametrize("out", [torch.float32, torch.float16, torch.bfloat16], ids=str)
@pytest.mark.parametrize("case", CASES, ids=[f"{i}" for i in range(len(CASES))])
def test_int4(ifa, case, out):
    B, Hkv, G, Nq, Nk, d, w, sinks, lens = case
    s = ref.problem(7, B, Hkv, G, Nq, Nk, d)
    want, tol = ref.attention(s, out, lens, w, sinks)
    check(int4(ifa, s, w, sinks, lens, out_dtype=out), want, tol)
