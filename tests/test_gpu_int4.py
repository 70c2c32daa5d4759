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


# (long: fp16 out alone)
LONG = [
    (1, 2, 8, 3, 700, 128, None, 0, None),               # 24 rows, eight wavefronts
    (1, 2, 4, 1, 600, 64, None, 0, (555,)),
    (2, 2, 4, 1, 800, 128, None, 0, (800, 333)),
    (3, 2, 9, 2, 500, 64, None, 0, (500, 320, 64)),
    (2, 1, 20, 1, 4000, 64, 3000, 3, (4000, 2222)),      # 20 rows, in parts
    (1, 3, 4, 1, 20000, 128, None, 0, None),             # more parts than 8
    (1, 1, 2, 1, 30000, 64, None, 0, (29999,)),
    (2, 32, 1, 600, 1500, 128, None, 0, (1500, 1111)),   # tiles of 128 rows
    (1, 4, 1, 512, 9000, 128, None, 0, None),            # ... in parts
    (2, 40, 1, 700, 900, 64, 700, 5, (900, 640)),
    (2, 20, 1, 256, 8000, 64, None, 0, (8000, 200)),
    (36, 2, 4, 64, 64, 128, None, 0, tuple(range(29, 65))),
    (150, 4, 1, 20, 40, 128, None, 0, tuple(b % 43 for b in range(150))),                 # ... of few rows, on short keys
    (90, 3, 3, 15, 300, 64, 100, 2, tuple(3 * b for b in range(90))),
]
# Parts by the lengths: more sequences than lanes, empty ones, one long
UNEVEN = [
    (64, 2, 1, 1, 3500, 64, None, 0, tuple((37 * b * b) % 3501 for b in range(64))),
    (70, 1, 2, 1, 6000, 128, None, 0, tuple(0 if b % 3 else 85 * b for b in range(70))),
    (16, 4, 3, 1, 7000, 128, None, 0, (7000,) + (100,) * 14 + (1,)),
    (16, 2, 8, 5, 6500, 64, None, 0, tuple(6500 * b // 15 for b in range(16))),       # 40 rows
    (24, 2, 20, 1, 9000, 128, 8000, 70, (9000, 8999, 3) + tuple(range(0, 2100, 100))),
    (12, 8, 4, 1, 5000, 64, None, 0, (0,) * 12),
]


@pytest.mark.parametrize("case", LONG + UNEVEN, ids=[f"long {i}" for i in range(len(LONG))] + [f"uneven {i}" for i in range(len(UNEVEN))])
def test_long(ifa, case):
    B, Hkv, G, Nq, Nk, d, w, sinks, lens = case
    s = ref.problem(11, B, Hkv, G, Nq, Nk, d)
    want, tol = ref.attention(s, torch.float16, lens, w, sinks)
    check(int4(ifa, s, w, sinks, lens), want, tol)


@pytest.mark.parametrize("out", [torch.float32, torch.float16, torch.bfloat16], ids=str)
@pytest.mark.parametrize("case", CASES, ids=[f"{i}" for i in range(len(CASES))])
def test_int4(ifa, case, out):
    B, Hkv, G, Nq, Nk, d, w, sinks, lens = case
    s = ref.problem(7, B, Hkv, G, Nq, Nk, d)
    want, tol = ref.attention(s, out, lens, w, sinks)
    check(int4(ifa, s, w, sinks, lens, out_dtype=out), want, tol)


# One of each kernel: few rows whole, in eight wavefronts, in parts, by lengths; tiles
KINDS = {
    "whole": (2, 2, 3, 1, 200, 128), "eight wavefronts": (2, 2, 3, 2, 600, 64), "in parts": (2, 2, 4, 2, 3000, 128), "by lengths": (64, 2, 2, 1, 3400, 64), "32 rows": (1, 2, 5, 5, 250, 64),
    "tiles": (2, 40, 1, 512, 1000, 64), "tiles in parts": (2, 8, 1, 256, 9000, 128)}


def of_kind(kind, seed=5):
    B, Hkv, G, Nq, Nk, d = KINDS[kind]
    return ref.problem(seed, B, Hkv, G, Nq, Nk, d), [Nk - (b * 13) % (Nk // 2) for b in range(B)]


@pytest.mark.parametrize("kind", KINDS)
def test_what_no_query_sees_is_not_looked_at(ifa, kind):
    """NaN and infinities in the scales behind L_b and, where every query is past it, in front of the window."""
    s, lens = of_kind(kind)
    B, Hkv, _, Nk = s["k4"].shape[0], s["k4"].shape[1], 0, s["k4"].shape[2]
    Nq, w, sinks = s["q8"].shape[2], 100, 3
    clean, tol = ref.attention(s, torch.float16, lens, w, sinks)
    for bad in (math.nan, math.inf, -3e38):
        for b in range(B):
            hidden = torch.ones(Nk, dtype=torch.bool)
            hidden[max(0, lens[b] - Nq - w + 1):lens[b]] = False
            hidden[:sinks] = False
            s["sk"][b][:, hidden] = bad
            s["sv"][b][:, hidden] = bad
        check(int4(ifa, s, w, sinks, lens), clean, tol)


@pytest.mark.parametrize("kind", KINDS)
def test_padding_queries_give_zeros_whatever_they_hold(ifa, kind):
    s, lens = of_kind(kind)
    Nq = s["q8"].shape[2]
    lens[0] = Nq // 2
    for bad in (0.0, math.nan, math.inf):
        s["sq"][0, :, :Nq - lens[0]] = bad
        s["sq"][1:, :, :] = s["sq"][1:, :, :].abs()
        clean = dict(s, sq=torch.nan_to_num(s["sq"], nan=1.0, posinf=1.0))
        want, tol = ref.attention(clean, torch.float16, lens)
        assert not want[0, :, :Nq - lens[0]].any()
        check(int4(ifa, s, None, 0, lens), want, tol)


@pytest.mark.parametrize("kind", KINDS)
def test_scales(ifa, kind):
    """s_Q = 0: all keys alike.  s_K of either sign and 0.  s_V of either sign, 0, apart by 2^40, all of them tiny or huge."""
    s, lens = of_kind(kind)
    g = torch.Generator().manual_seed(1)
    sign = torch.randint(0, 2, s["sk"].shape, generator=g) * 2.0 - 1.0
    zero = torch.rand(s["sk"].shape, generator=g) < 0.1
    spread = torch.exp2(torch.rand(s["sv"].shape, generator=g) * 20 - 10)
    one = dict(s, sq=s["sq"].clone(), sk=s["sk"] * sign * ~zero, sv=s["sv"] * sign.flip(2) * ~zero.flip(2) * spread)
    one["sq"][:, ::2] = 0.0
    for v in (one, dict(s, sv=s["sv"] * 2.0 ** -70), dict(s, sv=s["sv"] * 2.0 ** 60), dict(s, sv=torch.zeros_like(s["sv"]))):
        big = v["sv"].abs().max().item() > 1e4
        out = torch.float32 if big or v["sv"].abs().max().item() < 1e-9 else torch.float16
        want, tol = ref.attention(v, out, lens)
        check(int4(ifa, v, None, 0, lens, out_dtype=out), want, tol)


@pytest.mark.parametrize("kind", KINDS)
def test_scales_at_both_ends_of_their_range(ifa, kind):
    """s_V just below 2^20 beside 0, beside less than counts and beside 2^-20: the sum of the weights has every key in it, whichever comes first."""
    s, lens = of_kind(kind)
    g = torch.Generator().manual_seed(2)
    ends = torch.tensor([2.0 ** 20 * (1 - 2.0 ** -23), 0.0, 2.0 ** -90, -2.0 ** -20])
    for turn in (ends, ends.flip(0)[:3]):
        which = torch.randint(0, len(turn), s["sv"].shape, generator=g)
        which[:, :, :s["sv"].shape[2] // 2] = len(turn) - 1          # the first half alike, and among the smallest or the largest
        v = dict(s, sv=turn[which])
        want, tol = ref.attention(v, torch.float32, lens)
        check(int4(ifa, v, None, 0, lens, out_dtype=torch.float32), want, tol)


@pytest.mark.parametrize("kind", KINDS)
def test_a_key_of_all_the_weight_beside_large_values(ifa, kind):
    """The key that draws all the weight has values 2^-20 of its neighbours': the weights' range follows the products."""
    s, lens = of_kind(kind)
    s["k4"][:] = 0x88                                    # codes 0: scores 0
    s["k4"][:, :, 1] = 0xff                              # ... but for key 1, which every query sees
    s["q8"][:] = 100
    s["sq"][:], s["sk"][:] = 1.0, 0.0005                 # score 700 x 64 (128) x .0005 = 22 (45)
    s["sv"][:] = 1.0
    s["sv"][:, :, 1] = 2.0 ** -20
    want, tol = ref.attention(s, torch.float32, lens)
    check(int4(ifa, s, None, 0, lens, out_dtype=torch.float32), want, tol)


def test_a_long_rest_of_small_weights_counts(ifa):
    """One key 2^20 above all others, which together weigh 1 % of it, and all of the values."""
    for B, Hkv, Nq, Nk, d in ((1, 1, 1, 12000, 64), (2, 8, 256, 9000, 128)):
        s = ref.problem(3, B, Hkv, 1, Nq, Nk, d)
        s["q8"][:], s["k4"][:] = 10, 0x88
        s["k4"][:, :, 0] = 0x99                          # a score of d 10 s_Q s_K = 20 log 2
        s["sq"][:], s["sk"][:] = 20 * math.log(2) / (10 * d), 1.0
        s["sv"][:] = 1.0
        s["v4"][:] = 0xff
        s["v4"][:, :, 0] = 0x88
        want, tol = ref.attention(s, torch.float32)
        tol = torch.minimum(tol, want.abs() * 0.02)
        check(int4(ifa, s, out_dtype=torch.float32), want, tol)


@pytest.mark.parametrize("kind", KINDS)
def test_equal_calls_give_equal_bits(ifa, kind):
    s, lens = of_kind(kind)
    a = int4(ifa, s, 150, 2, lens, out_dtype=torch.float32)
    for _ in range(3):
        assert torch.equal(a, int4(ifa, s, 150, 2, lens, out_dtype=torch.float32))


@pytest.mark.parametrize("kind", KINDS)
def test_given_outputs_and_workspaces(ifa, kind):
    """Workspaces hold whatever: of a given size, larger ones, with any bytes in them; outputs of each type."""
    s, lens = of_kind(kind)
    t = ref.on_gpu(s)
    B, H, Nq, d = s["q8"].shape
    Hkv, Nk = s["k4"].shape[1:3]
    need = ifa.int4_workspace_bytes(B, H, Hkv, Nq, Nk, d)
    want = int4(ifa, s, None, 0, lens, out_dtype=torch.bfloat16)
    for fill in (0, 255):
        for n in (need, need + 4096):
            ws = torch.full((max(n, 1),), fill, dtype=torch.uint8, device="cuda")
            out = torch.full((B, H, Nq, d), 7.0, dtype=torch.bfloat16, device="cuda")
            call = lambda **kw: ifa.int_flash_attn_fwd_int4(t["q8"], t["k4"], t["v4"], t["sq"], t["sk"], t["sv"], lens=dev_lens(lens), workspace=ws, **kw)  # noqa: E731
            assert call(out=out) is out and torch.equal(out, want)
            assert torch.equal(call(out_dtype=torch.bfloat16), want)
    if need:
        with pytest.raises(ifa.IntfaError, match="WORKSPACE"):
            ifa.int_flash_attn_fwd_int4(t["q8"], t["k4"], t["v4"], t["sq"], t["sk"], t["sv"], lens=dev_lens(lens), workspace=torch.empty(need - 1, dtype=torch.uint8, device="cuda"))
