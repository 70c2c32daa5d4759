"""Calls on caches that do not fit the chip's own (past 64 MB they are read with the non-temporal hint) and on more heads than CUs, some of the heads against the definitions in 64 bits."""
import pytest
import torch

import cache_reference as ref
import cache_routes

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ifa():
    import paper_2409_16997_amd as ifa
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return ifa


def problem(B, Hkv, G, Nq, Nk, d, v, lens):
    """As cache_reference's, drawn on the GPU."""
    g = torch.Generator(device="cuda").manual_seed(5)

    def codes(*shape):
        return torch.randint(-127, 128, shape, generator=g, device="cuda", dtype=torch.int8)

    def scales(*shape):
        return (torch.rand(shape, generator=g, device="cuda") + 0.5) * (2.0 / (73.3 * 73.3 * d ** 0.5)) ** 0.5

    s = {"q8": codes(B, Hkv * G, Nq, d), "sq": scales(B, Hkv * G, Nq), "k8": codes(B, Hkv, Nk, d), "sk": scales(B, Hkv, Nk)}
    if v == "fp16":
        s["v"], s["sv"] = torch.randn((B, Hkv, Nk, d), generator=g, device="cuda").half(), None
    else:
        s["v"], s["sv"] = codes(B, Hkv, Nk, d), torch.rand((B, Hkv), generator=g, device="cuda") * 0.015 + 0.005
    return s, None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")


def head(s, b, hk, G):
    """Key head hk of sequence b and its queries, on the CPU."""
    own = {"q8": s["q8"][b:b + 1, hk * G:(hk + 1) * G], "sq": s["sq"][b:b + 1, hk * G:(hk + 1) * G]}
    own.update({k: None if s[k] is None else s[k][b:b + 1, hk:hk + 1] for k in ("k8", "sk", "v", "sv")})
    return {k: None if x is None else x.cpu() for k, x in own.items()}


# B, Hkv, G, Nq, Nk of d = 128 and fp16 V, lens; tiles copied ahead, past the caches.  (d = 64 and INT8 V: as many more keys.)
CASES = {
    "one ahead, past the caches": (3, 100, 2, 1, 800, (800, 131, 799), 1, True),
    "two ahead, past the caches": (2, 32, 4, 1, 3000, (3000, 2050), 2, True),
    "one ahead": (5, 100, 1, 3, 90, (90, 89, 1, 0, 33), 1, False),
}


@pytest.mark.parametrize("v", ["fp16", "int8"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("name", CASES)
def test_window(ifa, name, d, v):
    B, Hkv, G, Nq, Nk, lens, ahead, once = CASES[name]
    if once:
        k = (128 // d) * (3 if v == "int8" else 2)
        Nk, lens = Nk * k // 2, [n * k // 2 for n in lens]
    w, sinks = Nk - Nk // 20, 3
    plan = cache_routes.attention(B, Hkv, G, Nq, Nk, d, w, sinks, v=v)
    assert (plan["way"], plan["ahead"], plan["once"]) == ("few", ahead, once)
    s, ln = problem(B, Hkv, G, Nq, Nk, d, v, lens)
    got = ifa.int_flash_attn_fwd_window(s["q8"], s["k8"], s["v"], s["sq"], s["sk"], w, sinks, s_V=s["sv"], lens=ln, out_dtype=torch.float32)
    assert bool(torch.isfinite(got).all())
    for b, hk in ((0, 0), (B - 1, Hkv - 1), (1, Hkv // 2)):
        want, tol = ref.attention(head(s, b, hk, G), torch.float32, (lens[b],), w, sinks)
        off = (got[b:b + 1, hk * G:(hk + 1) * G].cpu().double() - want).abs()
        assert bool((off <= tol).all()), f"sequence {b}, head {hk}: off by up to {(off / tol.clamp_min(1e-300)).max().item():.3f} of the tolerance"


@pytest.mark.parametrize("d,rows,stored", [(64, 12, True), (64, 13, False), (128, 16, True), (128, 17, False)])
def test_key_weights_on_both_sides_of_the_stored_scores(ifa, d, rows, stored):
    assert cache_routes.weights(2, 2, rows, 1, 700, d)["stored"] == stored
    for G, Nq in ((rows, 1), (1, rows)):
        lens = (700, rows - 1)
        s = ref.problem(55, 2, 2, G, Nq, 700, d)
        want, tol = ref.key_weights(s, lens)
        t = ref.on_gpu(s)
        got = ifa.key_weights(t["q8"], t["k8"], t["sq"], t["sk"], lens=torch.tensor(lens, dtype=torch.int32, device="cuda"))
        off = (got.cpu().double() - want).abs()
        assert bool((off <= tol).all()), f"off by up to {(off / tol).max().item():.3f} of the tolerance"


@pytest.mark.parametrize("d,Nk", [(128, 8300), (64, 16700)])
def test_key_weights_past_the_caches(ifa, d, Nk):
    B, Hkv, G, lens = 2, 32, 4, (Nk, Nk // 3)
    plan = cache_routes.weights(B, Hkv, G, 1, Nk, d)
    assert plan["stored"] and plan["few"] and plan["once"]
    s, ln = problem(B, Hkv, G, 1, Nk, d, "int8", lens)
    W = torch.rand((B, Hkv, Nk), device="cuda")
    got = ifa.key_weights(s["q8"], s["k8"], s["sq"], s["sk"], W=W, lens=ln)
    for b, hk in ((0, 0), (1, 31), (1, 7)):
        want, tol = ref.key_weights(head(s, b, hk, G), (lens[b],), W[b:b + 1, hk:hk + 1].cpu())
        off = (got[b:b + 1, hk:hk + 1].cpu().double() - want).abs()
        assert bool((off <= tol).all()), f"sequence {b}, head {hk}: off by up to {(off / tol).max().item():.3f} of the tolerance"
