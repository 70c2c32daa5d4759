"""A sequence that goes on after its cache was cut down, as a program uses the calls together: prompt, key weights, eviction, room behind what is left, and steps that append a key each."""
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


def close(got, want, tol):
    off = (got.cpu().double() - want).abs()
    assert bool((off <= tol).all()), f"off by up to {(off / tol.clamp_min(1e-300)).max().item():.3f} of the tolerance"


@pytest.mark.parametrize("v", ["fp16", "int8"])
def test_steps_behind_an_eviction(ifa, v):
    B, Hkv, G, N, d, keep, room = 2, 2, 2, 300, 64, 96, 8
    lens = (300, 70)                                     # the second keeps all of its keys
    s = ref.problem(50, B, Hkv, G, N, N, d, v=v)
    t, ln = ref.on_gpu(s), torch.tensor(lens, dtype=torch.int32, device="cuda")
    k8, sk, V, sv = t["k8"], t["sk"], t["v"], t["sv"]

    O = ifa.int_flash_attn_fwd_window(t["q8"], k8, V, t["sq"], sk, window=N, s_V=sv, lens=ln)
    close(O, *ref.attention(s, torch.float16, lens))
    W = ifa.key_weights(t["q8"], k8, t["sq"], sk, lens=ln)
    close(W, *ref.key_weights(s, lens))
    k8, sk, V, W, index, ln = ifa.evict_keys(k8, sk, V, W, keep=keep, recent=20, sinks=4, lens=ln)
    assert ln.tolist() == [96, 70]

    pad = torch.nn.functional.pad
    k8, V, sk, W = pad(k8, (0, 0, 0, room)), pad(V, (0, 0, 0, room)), pad(sk, (0, room)), pad(W, (0, room))
    rows = torch.arange(B, device="cuda")
    host = {"k8": k8.cpu(), "sk": sk.cpu(), "v": V.cpu(), "sv": s["sv"]}
    weight = W.cpu().double()
    weight_tol = torch.zeros_like(weight)
    for step in range(room):
        new = ref.problem(60 + step, B, Hkv, G, 1, 1, d, v=v)
        q, n = ref.on_gpu({"q8": new["q8"], "sq": new["sq"]}), ref.on_gpu({k: new[k] for k in ("k8", "sk", "v")})
        at = ln.long()
        k8[rows, :, at], sk[rows, :, at], V[rows, :, at] = n["k8"][:, :, 0], n["sk"][:, :, 0], n["v"][:, :, 0]
        ln += 1
        O = ifa.int_flash_attn_fwd_window(q["q8"], k8, V, q["sq"], sk, window=k8.shape[2], s_V=sv, lens=ln)
        ifa.key_weights(q["q8"], k8, q["sq"], sk, W=W, lens=ln, out=W)
        # the same on the host
        now = (96 + step + 1, 70 + step + 1)
        for b in range(B):
            for k, x in (("k8", new["k8"]), ("sk", new["sk"]), ("v", new["v"])):
                host[k][b, :, now[b] - 1] = x[b, :, 0]
        whole = dict(host, q8=new["q8"], sq=new["sq"])
        close(O, *ref.attention(whole, torch.float16, now))
        more, tol = ref.key_weights(whole, now)
        weight, weight_tol = weight + more, weight_tol + tol + 2.0 ** -24 * (weight + more)      # an addition to W in fp32
        close(W, weight, weight_tol)
    again = ifa.evict_keys(k8, sk, V, W, keep=keep, recent=20, sinks=4, lens=ln)
    assert again[5].tolist() == [96, 78]


@pytest.mark.parametrize("case", [(2, 2, 1, 1, 300, 40, 64), (3, 1, 4, 1, 700, 65, 128), (40, 1, 4, 1, 2000, 200, 64), (3, 8, 2, 100, 70, 100, 128), (2, 4, 3, 200, 1000, 300, 64)], ids=str)
def test_prefix_into_given_tensors(ifa, case):
    """out= (the path through ctypes) and the caller's workspace: the same bits as the call that allocates, and nothing beside them."""
    B, Hkv, G, Nq, Np, Nk, d = case
    t = ref.on_gpu(ref.problem(51, B, Hkv, G, Nq, Nk, d, Np=Np))
    args = (t["q8"], t["kp8"], t["vp"], t["k8"], t["v"], t["sq"], t["skp"], t["sk"])
    for dtype in (torch.float16, torch.bfloat16, torch.float32):
        want = ifa.int_flash_attn_fwd_prefix(*args, out_dtype=dtype)
        out = torch.full((3, B, Hkv * G, Nq, d), 7.0, dtype=dtype, device="cuda")
        need = ifa.prefix_workspace_bytes(B, Hkv * G, Hkv, Nq, Np, Nk, d)
        ws = torch.full((need + 512,), 0xa5, dtype=torch.uint8, device="cuda")
        got = ifa.int_flash_attn_fwd_prefix(*args, out=out[1], workspace=ws[:need] if need else None)
        assert got.data_ptr() == out[1].data_ptr() and torch.equal(got, want)
        assert bool((out[0] == 7).all()) and bool((out[2] == 7).all()) and bool((ws[need:] == 0xa5).all())
        assert torch.equal(ifa.int_flash_attn_fwd_prefix(*args, out=out[2]), want)
