"""append_keys, read_keys and int_flash_attn_fwd_int4 through the binding's native module and on the general path behind it: the same results and the same refusals."""
import pytest

torch = pytest.importorskip("torch")

import append_reference as written  # noqa: E402
from test_gpu_host_calls import general, tensors  # noqa: E402

pytestmark = pytest.mark.gpu


def state(held, B=2, Hkv=3, G=2, Nq=2, Nk=50, d=64, dtype=torch.float16):
    import paper_2409_16997_amd as ifa
    g = torch.Generator(device="cuda").manual_seed(Nk)
    r = lambda *s: torch.randn(s, device="cuda", generator=g)  # noqa: E731
    sv = torch.rand(B, Hkv, device="cuda", generator=g) * 0.1 + 0.01 if held == "i8" else None
    cache = [None if x is None else x.cuda() for x in written.empty_cache(held, B, Hkv, Nk, d, sv)]
    K, V = r(B, Nk, Hkv, d).to(dtype).transpose(1, 2), r(B, Hkv, Nk, d).to(dtype)
    ifa.append_keys(K, V, *cache)
    q8, sq = ifa.quantize_tokenwise(r(B, Hkv * G, Nq, d), scale_mul=d ** -0.5)
    lens = torch.tensor([Nk - 11 * b for b in range(B)], dtype=torch.int32, device="cuda")
    return {"K": K[:, :, :7], "V": V[:, :, :7], "cache": cache, "q8": q8, "sq": sq, "lens": lens}


def appended(ifa, s, **kw):
    cache = [None if x is None else x.clone() for x in s["cache"]]
    assert ifa.append_keys(s["K"], s["V"], *cache, **kw) is None
    return tuple(x for x in cache if x is not None)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16, torch.float32], ids=str)
@pytest.mark.parametrize("held", ["i4", "i8", "i8f16"])
def test_both_paths_agree(held, dtype):
    import paper_2409_16997_amd as ifa
    from paper_2409_16997_amd import binding
    assert not isinstance(binding._load_native(), binding._NoNative)
    s = state(held, dtype=dtype)
    c, ln = s["cache"], s["lens"]
    calls = [lambda h=h, n=n: appended(ifa, s, lens=n, hadamard=h) for h in (False, True) for n in (None, ln)]
    calls += [lambda f=f, n=n, t=t: ifa.read_keys(*c, lens=n, first=f, count=9, hadamard=True, out_dtype=t) for f in (0, 45, None) for n in (None, ln) for t in (None, dtype)]
    calls += [lambda: ifa.read_keys(*c), lambda: ifa.read_keys(*c, first=3), lambda: ifa.read_keys(*c, first=None), lambda: ifa.read_keys(*c, first=None, lens=ln)]
    if held == "i4":
        calls += [lambda w=w, n=n, t=t: ifa.int_flash_attn_fwd_int4(s["q8"], c[0], c[2], s["sq"], c[1], c[3], window=w, sinks=2, lens=n, out_dtype=t)
                  for w in (None, 10, 1 << 40) for n in (None, ln) for t in (None, torch.float32)]
    for i, f in enumerate(calls):
        a, b = tensors(f()), tensors(general(f))
        assert len(a) == len(b) > 0, i
        for x, y in zip(a, b):
            assert x.dtype is y.dtype and x.shape == y.shape and x.stride() == y.stride() and torch.equal(x, y), i
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = [tensors(f()) for f in calls]
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(p, q) for x, f in zip(got, calls) for p, q in zip(x, tensors(f())))


def test_refusals_are_those_of_the_general_path(monkeypatch):
    import paper_2409_16997_amd as ifa
    s = state("i4")
    c, q8, sq, K, V = s["cache"], s["q8"], s["sq"], s["K"], s["V"]
    e = state("i8")["cache"]
    app, read = ifa.append_keys, ifa.read_keys
    def att(q=q8, k=c[0], v=c[2], a=sq, b=c[1], d=c[3], **kw):  # noqa: E306
        return ifa.int_flash_attn_fwd_int4(q, k, v, a, b, d, **kw)
    wide = torch.zeros(2, 3, 7, 128, device="cuda").half()
    bad = [lambda: app(K.cpu(), V, *c), lambda: app(K, V.float(), *c), lambda: app(K, V[:, :, :3], *c), lambda: app(K[:, :, :0], V[:, :, :0], *c), lambda: app(K.double(), V.double(), *c),
           lambda: app(wide[..., ::2], V, *c), lambda: app(wide[..., 1:65], V, *c), lambda: app(K, V, *c[:3]), lambda: app(K, V, c[0], c[1], c[2], c[3][:, :, :5]), lambda: app(K, V, c[0].view(torch.int8), *c[1:]),
           lambda: app(K, V, *e[:3], c[3]), lambda: app(K, V, c[0][:, :, ::2], *c[1:]), lambda: app(K, V, *c, lens=s["lens"].long()), lambda: app(K, V, *c, lens=s["lens"][:1]), lambda: app(K, V, None, *c[1:]),
           lambda: app(c[0].view(torch.float16)[:, :, :7, :16].expand(2, 3, 7, 16), V, *c), lambda: app(K, V, c[0], c[1], c[0], c[3]), lambda: app(K, V, c[0], c[1], c[2], c[1]),
           lambda: app(c[0].view(torch.float16).flatten()[:2 * 3 * 7 * 64].view(2, 3, 7, 64), V, *c),
           lambda: read(*c, first=51), lambda: read(*c, first=-2), lambda: read(*c, count=0), lambda: read(*c, first=50), lambda: read(*c, out_dtype=torch.float64), lambda: read(c[0], c[1], e[2], c[3]),
           lambda: read(*c, out=(V, V)), lambda: read(*c, count=1 << 40), lambda: read(*c, count=1 << 27),
           lambda: att(q=q8[..., :32].contiguous()), lambda: att(k=e[0]), lambda: att(d=e[3]), lambda: att(window=0), lambda: att(sinks=-1), lambda: att(q=q8[:, :5].contiguous(), a=sq[:, :5].contiguous()),
           lambda: att(a=sq.double()), lambda: att(lens=s["lens"].cpu()), lambda: att(out_dtype=torch.int8), lambda: att(workspace=torch.empty(8, dtype=torch.float32, device="cuda")), lambda: att(q=None),
           lambda: att(q=q8[0]), lambda: att(q=q8[:, :, :0])]
    for i, f in enumerate(bad):
        seen = []
        for path in (lambda: f(), lambda: general(f)):
            with pytest.raises(Exception) as err:
                path()
            seen.append((err.type, str(err.value)))
        assert seen[0] == seen[1], (i, seen)
        assert "out of memory" not in seen[0][1], i
    for i, f in enumerate(bad[-2:]):
        with pytest.raises(ifa.IntfaError):
            f()
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)     # tensors of another device than the current one: the general path says so
    for f in (lambda: app(K, V, *c), lambda: read(*c), lambda: att()):
        with pytest.raises(ifa.IntfaError, match="current device is cuda:1"):
            general(f)


def test_a_hip_error_is_raised_and_the_call_not_repeated():
    import ctypes
    from paper_2409_16997_amd import binding as ifa
    s = state("i4")
    c = s["cache"]
    calls = [lambda: ifa.append_keys(s["K"], s["V"], *c), lambda: ifa.read_keys(*c, count=5),
             lambda: ifa.int_flash_attn_fwd_int4(s["q8"], c[0], c[2], s["sq"], c[1], c[3])]
    fail = ctypes.CFUNCTYPE(ctypes.c_int)(lambda: -5)            # IFA_ERR_HIP
    module = ifa._load_native()
    addresses = [ifa._address(getattr(ifa.lib(), name)) for name in ifa._NATIVE_CALLS]
    stand_in = [ifa._address(fail) if name in ("append_keys", "read_keys", "int_flash_attn_fwd_int4") else a for name, a in zip(ifa._NATIVE_CALLS, addresses)]
    try:
        module.init(ifa._check, *stand_in)
        for f in calls:
            with pytest.raises(ifa.IntfaError, match="IFA_ERR_HIP"):
                f()
    finally:
        module.init(ifa._check, *addresses)
    for f in calls:
        f()
