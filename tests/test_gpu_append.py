"""Tokens written into a quantized cache and read back, bit for bit against the definition."""
import pytest
import torch

import append_reference as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ifa():
    import paper_2409_16997_amd as ifa
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return ifa


def gpu(x):
    return None if x is None else x.cuda()


def dev_lens(lens):
    return None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")


def same(got, want):
    for name, g, w in zip(("K", "s_K", "V", "s_V"), got, want):
        if w is not None:
            equal = torch.equal(g.cpu().contiguous().view(torch.uint8), w.contiguous().view(torch.uint8))
            assert equal, f"{name}: {(g.cpu() != w).sum().item()} of {w.numel()} differ"


def tokens(seed, B, Hkv, Nn, d, dtype):
    g = torch.Generator().manual_seed(seed)
    scale = torch.exp(torch.randn(B, Hkv, Nn, 1, generator=g) * 2)
    return [(torch.randn(B, Hkv, Nn, d, generator=g) * scale).to(dtype) for _ in range(2)]


def v_scale(held, B, Hkv):
    return torch.linspace(0.01, 0.1, B * Hkv).view(B, Hkv) if held == "i8" else None


# B, Hkv, Nn, Nk, d, lens
CASES = [
    (1, 1, 1, 1, 64, None),
    (2, 3, 1, 33, 128, (33, 1)),                         # a step; the first key
    (3, 2, 5, 40, 64, (40, 0, 3)),                       # nothing there, padding in front
    (1, 4, 300, 300, 128, None),                         # a prompt that fills the cache
    (2, 5, 257, 1000, 64, (700, 100)),
    (4, 1, 70, 50, 128, (50, 7, -2, 90)),                # more tokens than slots, lengths out of range
    (64, 8, 1, 100, 128, tuple(range(1, 65))),
    (2, 9, 2000, 2100, 64, (2100, 1999)),                # several rows to a thread
    (1, 7, 2500, 2600, 128, (2555,)),
]
DTYPES = [torch.float16, torch.bfloat16, torch.float32]


@pytest.mark.parametrize("held", ["i4", "i8", "i8f16"])
@pytest.mark.parametrize("dtype", DTYPES, ids=str)
@pytest.mark.parametrize("case", CASES, ids=[f"{i}" for i in range(len(CASES))])
def test_append(ifa, case, dtype, held):
    B, Hkv, Nn, Nk, d, lens = case
    K, V = tokens(Nn + d, B, Hkv, Nn, d, dtype)
    cache = ref.empty_cache(held, B, Hkv, Nk, d, v_scale(held, B, Hkv))
    for rotated in (False, True):
        here = [gpu(x) for x in cache]
        ifa.append_keys(K.cuda(), V.cuda(), *here, lens=dev_lens(lens), hadamard=rotated)
        same(here, ref.append(held, K, V, cache, lens, rotated))


@pytest.mark.parametrize("held", ["i4", "i8", "i8f16"])
@pytest.mark.parametrize("dtype", DTYPES, ids=str)
@pytest.mark.parametrize("d", [64, 128])
def test_read(ifa, d, dtype, held):
    B, Hkv, Nk = 3, 5, 300
    g = torch.Generator().manual_seed(d)
    lens = (300, 77, 0)
    cache = ref.empty_cache(held, B, Hkv, Nk, d, v_scale(held, B, Hkv))
    for i in (0, 2):
        if cache[i].dtype != torch.float16:
            cache[i] = torch.randint(-128, 128, cache[i].shape, generator=g).to(torch.int8).view(cache[i].dtype)     # every code there is
        else:
            cache[i] = torch.randn(cache[i].shape, generator=g).half()
    cache[1] = torch.randn(B, Hkv, Nk, generator=g)
    if held == "i4":
        cache[3] = torch.randn(B, Hkv, Nk, generator=g)
    here = [gpu(x) for x in cache]
    for first, count in ((0, 300), (0, 1), (299, 1), (300, 5), (70, 20), (250, 60), (None, 1), (None, 90), (None, 300), (None, 301)):
        for ln in (None, lens):
            for rotated in (False, True):
                got = ifa.read_keys(*here, lens=dev_lens(ln), first=first, count=count, hadamard=rotated, out_dtype=dtype)
                same(got, ref.read(held, cache, ln, first, count, rotated, dtype))
    got = ifa.read_keys(*here, first=123, out_dtype=dtype)
    same(got, ref.read(held, cache, None, 123, 177, False, dtype))


def test_read_many_rows(ifa):
    """Several rows to a thread, the last workgroup cut."""
    for held, d, Nk in (("i4", 128, 9001), ("i8f16", 64, 9001)):
        K, V = tokens(5, 1, 2, Nk, d, torch.bfloat16)
        here = [gpu(x) for x in ref.empty_cache(held, 1, 2, Nk, d)]
        ifa.append_keys(K.cuda(), V.cuda(), *here)
        cache = [None if x is None else x.cpu() for x in here]
        for first in (0, None):
            got = ifa.read_keys(*here, first=first, count=Nk, out_dtype=torch.float32)
            if held == "i4":
                want = [ref.unpack(cache[0]) * cache[1][..., None], ref.unpack(cache[2]) * cache[3][..., None]]
            else:
                want = [cache[0].float() * cache[1][..., None], cache[2].float()]
            same(got, want)


@pytest.mark.parametrize("held", ["i4", "i8", "i8f16"])
def test_rows_that_are_hard_to_round(ifa, held):
    """Ties on every border, zeros, the smallest and the largest numbers of the type, one number alone."""
    d = 64
    rows = []
    for a in (7.0, 3.5, 127.0, 1.0):
        x = torch.linspace(-a, a, d)
        rows += [x, torch.cat([torch.arange(32) / 2 * a / 16, -torch.arange(32) / 2 * a / 16])]
    ties = torch.tensor([k + 0.5 for k in range(-7, 7)] * 4 + [7.0] * 8)
    one = torch.zeros(d)
    one[37] = -5.0
    rows += [ties, torch.zeros(d), one, -one]
    for dtype, extremes in ((torch.float16, (65504.0, 6e-8, 6.2e-5)), (torch.bfloat16, (3.3e38, 1e-30, 2.0 ** -117)), (torch.float32, (3.4e38, 2.0 ** -118, 2.0 ** -119, 1e-40))):
        x = torch.stack(rows + [ties / 7.0 * e for e in extremes if held == "i4" or 1e-30 <= e]).to(dtype)[None, None]
        n = x.shape[2]
        cache = ref.empty_cache(held, 1, 1, n, d, torch.tensor([[0.037]]) if held == "i8" else None)
        v = x if held == "i4" else x.float().clamp(-60000, 60000).to(dtype)
        here = [gpu(t) for t in cache]
        ifa.append_keys(x.cuda(), v.cuda(), *here)
        same(here, ref.append(held, x, v, cache, None, False))


def test_a_value_scale_of_zero(ifa):
    K, V = tokens(1, 1, 2, 3, 64, torch.float16)
    cache = ref.empty_cache("i8", 1, 2, 4, 64, torch.tensor([[0.0, 0.05]]))
    here = [gpu(x) for x in cache]
    ifa.append_keys(K.cuda(), V.cuda(), *here)
    same(here, ref.append("i8", K, V, cache, None, False))
    assert not here[2][0, 0, 1:].any()


def test_eight_bits_are_those_of_the_quantizers(ifa):
    for rotated in (False, True):
        K, V = tokens(3, 2, 3, 50, 128, torch.float16)
        q, s = ifa.quantize_tokenwise(K.cuda(), hadamard=rotated)
        here = [gpu(x) for x in ref.empty_cache("i8f16", 2, 3, 50, 128)]
        ifa.append_keys(K.cuda(), V.cuda(), *here, hadamard=rotated)
        assert torch.equal(here[0], q) and torch.equal(here[1], s) and torch.equal(here[2], V.cuda())


@pytest.mark.parametrize("dtype", DTYPES, ids=str)
def test_layouts(ifa, dtype):
    """Tokens as a projection leaves them: token by token, q, k and v of a token behind each other, one head for several, one row for several tokens."""
    B, Hkv, Nn, d = 2, 3, 37, 64
    wide = torch.randn(B, Nn, 3, 5, d, generator=torch.Generator().manual_seed(0)).to(dtype).cuda()
    K, V = wide[:, :, 1, 1:4].transpose(1, 2), wide[:, :, 2, 1:4].transpose(1, 2)
    narrow = torch.randn(B, Nn, 1, d + 24, generator=torch.Generator().manual_seed(1)).to(dtype).cuda()
    views = [(K, V), (K.contiguous(), V), (narrow[..., 8:72].transpose(1, 2).expand(B, Hkv, Nn, d), V), (K[:, :, :1].expand(B, Hkv, Nn, d), V[:, :1].expand(B, Hkv, Nn, d)),
             (K[::2, :, ::3], V[1:, :, ::3])]
    for k, v in views:
        n = k.shape[2]
        cache = ref.empty_cache("i4", k.shape[0], Hkv, 40, d)
        here = [gpu(x) for x in cache]
        ifa.append_keys(k, v, *here)
        same(here, ref.append("i4", k.cpu().contiguous(), v.cpu().contiguous(), cache, None, False))
        back = ifa.read_keys(*here, first=None, count=n, out_dtype=dtype)
        same(back, ref.read("i4", [x.cpu() for x in here], None, None, n, False, dtype))


def test_outputs_given(ifa):
    K, V = tokens(2, 1, 2, 30, 64, torch.float16)
    here = [gpu(x) for x in ref.empty_cache("i4", 1, 2, 30, 64)]
    ifa.append_keys(K.cuda(), V.cuda(), *here)
    out = tuple(torch.full((1, 2, 10, 64), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    got = ifa.read_keys(*here, first=20, count=10, out=out)
    assert got[0] is out[0] and got[1] is out[1]
    same(out, ref.read("i4", [x.cpu() for x in here], None, 20, 10, False, torch.bfloat16))
