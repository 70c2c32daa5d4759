"""Rows, heads and blocks so small that 127 / a, or 1 / s_V, is infinite: by the rule of the quantizers every number but 0 is then +-127 (the largest of them is, too, and none is off by more than it), and 0 is 0."""
import pytest
import torch

import append_reference as written
import oracle

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ifa():
    import paper_2409_16997_amd as ifa
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return ifa


def numbers(a, shape, dtype):
    """Numbers of at most `a` in magnitude, every third a zero of either sign, the largest in each row."""
    g = torch.Generator().manual_seed(1)
    x = (torch.rand(shape, generator=g) * 2 - 1) * a
    x[..., ::3] = 0.0
    x[..., 3::6] = -0.0
    x[..., 1] = a
    return x.to(dtype)


# below 127 / max fp32 = 3.7e-37: normal numbers, the smallest normal one, subnormal ones; and one just above
SIZES = [(torch.float32, 3.6e-37), (torch.bfloat16, 1e-37), (torch.float32, 2.0 ** -126), (torch.float32, 1e-40), (torch.float32, 3.8e-37)]
ids = [f"{t}-{a:g}" for t, a in SIZES]


def want(x):
    """(codes, scales) of rows."""
    a = x.float().abs().amax(-1)
    inv = torch.full_like(a, 127.0) / a
    q = torch.where(x.float() == 0, torch.zeros(()), x.float() * inv[..., None])
    return torch.round(q.clamp(-127, 127)).to(torch.int8), a / torch.full_like(a, 127.0)


@pytest.mark.parametrize("dtype,a", SIZES, ids=ids)
def test_rows(ifa, dtype, a):
    x = numbers(a, (2, 3, 40, 64), dtype)
    q, s = want(x)
    oq, _ = oracle.quantize_tokenwise(x.float().numpy())
    assert torch.equal(torch.from_numpy(oq).view(q.shape), q)
    for got in (ifa.quantize_tokenwise(x.cuda()), ifa.quantize_qk(x.cuda(), x.cuda())[1::2], ifa.quantize_qkv(x.cuda(), x.cuda(), x.cuda())[1::3]):
        assert torch.equal(got[0].cpu(), q) and torch.equal(got[1].cpu(), s)
    assert not q[..., ::3].any()


@pytest.mark.parametrize("dtype,a", SIZES, ids=ids)
def test_heads_and_blocks(ifa, dtype, a):
    for N in (32, 4000):                                             # one launch and two
        x = numbers(a, (1, 3, N, 64), dtype)
        q, s = want(x.flatten(2))
        for glob in (False, True):
            got = ifa.quantize_headwise(x.cuda(), global_scale=glob)
            assert torch.equal(got[0].cpu().flatten(2), q) and torch.equal(got[1].cpu(), s)
        got = ifa.quantize_qkv(x.cuda(), x.cuda(), x.cuda())
        assert torch.equal(got[2].cpu().flatten(2), q) and torch.equal(got[5].cpu(), s)
        got = ifa.quantize_blockwise(x.cuda(), 32)
        q, s = want(x.view(1, 3, N // 32, 32 * 64))
        assert torch.equal(got[0].cpu().view(q.shape), q) and torch.equal(got[1].cpu(), s)


@pytest.mark.parametrize("dtype,a", SIZES, ids=ids)
def test_tokens_into_the_cache(ifa, dtype, a):
    x = numbers(a, (2, 3, 40, 64), dtype)
    q, s = want(x)
    sv = torch.tensor([[a / 100, 1e-39, 2.0 ** -149], [0.0, 0.5, 2.0 ** -127]])
    for held in ("i8", "i8f16"):
        here = [None if t is None else t.cuda() for t in written.empty_cache(held, 2, 3, 40, 64, sv if held == "i8" else None)]
        ifa.append_keys(x.cuda(), x.cuda(), *here)
        assert torch.equal(here[0].cpu(), q) and torch.equal(here[1].cpu(), s)
    here = [t.cuda() for t in written.empty_cache("i8", 2, 3, 40, 64, sv)]
    ifa.append_keys(x.cuda(), x.cuda(), *here)
    inv = torch.where(sv == 0, 0.0, 1.0 / sv)[..., None, None]
    v = torch.where(x.float() == 0, torch.zeros(()), x.float() * inv)
    assert torch.equal(here[2].cpu(), torch.round(v.clamp(-127, 127)).to(torch.int8))
