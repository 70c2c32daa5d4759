"""Key weights and the eviction that goes by them, against their definitions in 64 bits, and the calls on a cache one after the other."""
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


def dev_lens(lens):
    return None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")


# B, Hkv, G, Nq, Nk, d, lens
WEIGHTS = [
    (1, 1, 1, 1, 1, 64, None),
    (2, 2, 1, 1, 33, 128, (33, 32)),
    (2, 3, 4, 1, 1500, 128, (1500, 1023)),
    (3, 1, 8, 2, 700, 64, (700, 0, 1)),                  # 16 rows: the most whose scores are stored; an empty sequence
    (1, 2, 17, 1, 600, 128, None),                       # 17: computed again
    (2, 1, 3, 6, 260, 64, (260, 4)),                     # more queries than keys
    (1, 2, 2, 40, 300, 128, (299,)),
    (1, 1, 1, 129, 129, 64, None),                       # a prompt
    (2, 2, 3, 200, 200, 128, (200, 130)),                # prompts, one padded in front
    (1, 1, 1, 64, 5000, 64, (4999,)),
    (1, 1, 2, 700, 900, 128, None),
    (2, 8, 2, 150, 1200, 128, (1200, 700)),              # tiles of 128 rows, the keys in parts
    (1, 20, 3, 80, 200, 64, (190,)),                     # ... in one
    (3, 2, 7, 11, 700, 128, (700, 13, 5)),               # a few queries of many heads, an odd group
    (2, 1, 4, 1, 20000, 64, (20000, 19999)),             # many parts of stored scores
    (5, 1, 1, 31, 31, 128, (31, 30, 1, 0, 16)),
]


@pytest.mark.parametrize("past", [False, True])
@pytest.mark.parametrize("case", WEIGHTS, ids=[f"{i}" for i in range(len(WEIGHTS))])
def test_key_weights(ifa, case, past):
    B, Hkv, G, Nq, Nk, d, lens = case
    s = ref.problem(11, B, Hkv, G, Nq, Nk, d)
    W = torch.rand(B, Hkv, Nk, generator=torch.Generator().manual_seed(1)) if past else None
    want, tol = ref.key_weights(s, lens, W)
    t = ref.on_gpu(s)
    w = None if W is None else W.cuda()
    got = ifa.key_weights(t["q8"], t["k8"], t["sq"], t["sk"], W=w, lens=dev_lens(lens))
    off = (got.cpu().double() - want).abs()
    assert bool((off <= tol).all()), f"off by up to {(off / tol).max().item():.3f} of the tolerance"
    if past:                                             # in place, and the same again
        again = ifa.key_weights(t["q8"], t["k8"], t["sq"], t["sk"], W=w, lens=dev_lens(lens), out=w)
        assert again.data_ptr() == w.data_ptr() and torch.equal(again, got)


def test_weights_of_what_lies_behind_the_sequence(ifa):
    """NaN in the codes' scales behind L_b; the weights there stay as they were."""
    for G, Nq in ((1, 1), (2, 30)):
        s = ref.problem(12, 1, 1, G, Nq, 400, 128)
        want, tol = ref.key_weights(s, (333,))
        s["sk"][:, :, 333:] = math.nan
        t = ref.on_gpu(s)
        W = torch.full((1, 1, 400), 0.25, device="cuda")
        got = ifa.key_weights(t["q8"], t["k8"], t["sq"], t["sk"], W=W, lens=dev_lens((333,))).cpu().double()
        assert bool(((got - want - 0.25).abs() <= tol + 2.0 ** -23 * (want + 0.25)).all()) and bool((got[:, :, 333:] == 0.25).all())


@pytest.mark.parametrize("Hkv,G,Nq", [(1, 1, 9), (1, 2, 30), (16, 2, 200)])   # stored scores, the kernel for 32 rows, tiles of 128
def test_what_padding_queries_hold_does_not_matter(ifa, Hkv, G, Nq):
    s = ref.problem(2, 1, Hkv, G, Nq, 260, 64)
    want, tol = ref.key_weights(s, (5,))
    for bad in (0.0, math.nan, math.inf):
        s["sq"][:, :, :Nq - 5] = bad
        t = ref.on_gpu(s)
        got = ifa.key_weights(t["q8"], t["k8"], t["sq"], t["sk"], lens=dev_lens((5,))).cpu().double()
        assert bool(((got - want).abs() <= tol).all())


# B, Hkv, Nk, d, keep, recent, sinks, lens
EVICTIONS = [
    (1, 1, 1, 64, 1, 0, 0, None),
    (2, 2, 33, 128, 32, 0, 0, None),
    (3, 2, 700, 64, 256, 32, 4, (700, 256, 0)),
    (1, 1, 5000, 128, 4999, 100, 0, None),
    (2, 1, 9000, 64, 1000, 0, 7, (9000, 1001)),          # several rounds of the workgroup
    (1, 3, 300, 128, 100, 60, 40, None),                 # nothing is chosen by weight
    (1, 1, 4097, 64, 4096, 0, 0, None),
    (1, 2, 260, 32, 37, 3, 2, (259,)),
    (1, 1, 40000, 16, 300, 7, 1, (39999,)),              # weights read again in each pass
    (1, 2, 32768, 16, 30000, 0, 4, (31000,)),            # the most that stay in registers
    (2, 1, 16384, 48, 16000, 0, 0, None),
]


@pytest.mark.parametrize("v", ["fp16", "int8"])
@pytest.mark.parametrize("weights", ["spread", "equal", "few values", "strange"])
@pytest.mark.parametrize("case", EVICTIONS, ids=[f"{i}" for i in range(len(EVICTIONS))])
def test_evict(ifa, case, weights, v):
    B, Hkv, Nk, d, keep, recent, sinks, lens = case
    s = ref.problem(13, B, Hkv, 1, 1, Nk, d, v=v)
    g = torch.Generator().manual_seed(2)
    W = torch.exp(3 * torch.randn(B, Hkv, Nk, generator=g))
    if weights == "equal":
        W = torch.full_like(W, 0.5)
    elif weights == "few values":
        W = torch.randint(0, 3, W.shape, generator=g).float() * 1e-3
    elif weights == "strange":                           # both zeros, negative ones, infinities, NaN, subnormals
        W = torch.tensor([0.0, -0.0, -1.5, math.inf, -math.inf, math.nan, 1e-42, 2e-42, -1e-42, 1.0])[torch.randint(0, 10, W.shape, generator=g)]
    want = ref.evict(s, W, keep, recent, sinks, lens)
    t = ref.on_gpu(s)
    got = ifa.evict_keys(t["k8"], t["sk"], t["v"], W.cuda(), keep, recent, sinks, lens=dev_lens(lens))
    for i, (a, b) in enumerate(zip(got, want)):
        assert a.dtype == b.dtype and torch.equal(a.cpu().nan_to_num(nan=-7.0) if a.is_floating_point() else a.cpu(), b.nan_to_num(nan=-7.0) if b.is_floating_point() else b), i


def test_evict_into_given_tensors_and_not_in_place(ifa):
    s = ref.on_gpu(ref.problem(14, 1, 1, 1, 1, 100, 64))
    W = torch.rand(1, 1, 100, device="cuda")
    fresh = ifa.evict_keys(s["k8"], s["sk"], s["v"], W, 40)
    big = torch.full((3, 1, 1, 40, 64), 9, dtype=torch.int8, device="cuda")
    out = (big[1],) + tuple(torch.empty_like(x) for x in fresh[1:])
    got = ifa.evict_keys(s["k8"], s["sk"], s["v"], W, 40, out=out)
    assert all(torch.equal(a, b) for a, b in zip(got, fresh)) and bool((big[0] == 9).all()) and bool((big[2] == 9).all())
    with pytest.raises(ifa.IntfaError, match="IFA_ERR_UNSUPPORTED"):
        ifa.evict_keys(s["k8"], s["sk"], s["v"], W, 40, out=(s["k8"].view(-1)[:40 * 64].view(1, 1, 40, 64),) + tuple(fresh[1:]))


def test_a_sequence_in_use(ifa):
    """A prompt through a window, its key weights, the eviction, then decode steps on what is left -- with a shared prefix, too -- against the same in 64 bits."""
    B, Hkv, G, N, d, keep, recent, sinks, Np = 2, 2, 2, 300, 64, 96, 20, 4, 130
    s = ref.problem(15, B, Hkv, G, N, N, d, Np=Np)
    own = {k: x for k, x in s.items() if not k.endswith("p") and not k.startswith("kp") and not k.startswith("vp") and not k.startswith("svp") and not k.startswith("skp")}
    t, lens = ref.on_gpu(s), (300, 211)
    ln = dev_lens(lens)
    O = ifa.int_flash_attn_fwd_window(t["q8"], t["k8"], t["v"], t["sq"], t["sk"], 128, sinks, lens=ln)
    want, tol = ref.attention(own, torch.float16, lens, 128, sinks)
    assert bool(((O.cpu().double() - want).abs() <= tol).all())
    W = ifa.key_weights(t["q8"], t["k8"], t["sq"], t["sk"], lens=ln)
    k8, sk, v, w, index, left = ifa.evict_keys(t["k8"], t["sk"], t["v"], W, keep, recent, sinks, lens=ln)
    cut = ref.evict(own, W.cpu(), keep, recent, sinks, lens)
    assert torch.equal(index.cpu(), cut[4]) and left.tolist() == [96, 96]
    step = ref.problem(16, B, Hkv, G, 1, keep, d)        # one new query each
    q, sq = step["q8"].cuda(), step["sq"].cuda()
    after = {"q8": step["q8"], "sq": step["sq"], "k8": cut[0], "sk": cut[1], "v": cut[2], "sv": None}
    want, tol = ref.attention(after, torch.float16, (96, 96), 10 ** 6)
    got = ifa.int_flash_attn_fwd_window(q, k8, v, sq, sk, keep, lens=left)
    assert bool(((got.cpu().double() - want).abs() <= tol).all())
    want, tol = ref.attention(dict(after, kp8=s["kp8"], skp=s["skp"], vp=s["vp"], svp=None), torch.float16, (96, 96))
    got = ifa.int_flash_attn_fwd_prefix(q, t["kp8"], t["vp"], k8, v, sq, t["skp"], sk, lens=left)
    assert bool(((got.cpu().double() - want).abs() <= tol).all())
    more = ifa.key_weights(q, k8, sq, sk, W=w, lens=left, out=w)
    want, tol = ref.key_weights(after, (96, 96), cut[3])
    assert bool(((more.cpu().double() - want).abs() <= tol).all())


def test_graph_replays(ifa):
    """Weights (both ways), eviction and a step on what is left in one captured graph, inputs changed between replays."""
    s, lens = ref.problem(17, 2, 2, 4, 1, 900, 128), (900, 400)
    t, ln = ref.on_gpu(s), dev_lens(lens)
    many = ref.on_gpu(ref.problem(18, 2, 2, 4, 30, 900, 128))
    W0 = torch.zeros(2, 2, 900, device="cuda")

    def step():
        W = ifa.key_weights(t["q8"], t["k8"], t["sq"], t["sk"], W=W0, lens=ln)
        W = ifa.key_weights(many["q8"], t["k8"], many["sq"], t["sk"], W=W, lens=ln)
        k8, sk, v, w, index, left = ifa.evict_keys(t["k8"], t["sk"], t["v"], W, 256, 16, 4, lens=ln)
        return W, k8, sk, v, w, index, left, ifa.int_flash_attn_fwd_window(t["q8"], k8, v, t["sq"], sk, 256, lens=left)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for k in range(3):
        t["q8"].copy_(torch.roll(t["q8"], 1, -1))
        ln.copy_(torch.tensor([900 - 11 * k, 100 * k], dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        eager = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(captured, eager))


def test_offsets_beyond_32_bits(ifa):
    """The last of 36 heads of 2^20 keys (4.8 GB of K, which is V, too): what it gives is what its last keys give in a cache of their own."""
    H, N, d = 36, 1 << 20, 128
    g = torch.Generator(device="cuda").manual_seed(3)
    k8 = torch.randint(-127, 128, (1, H, N, d), dtype=torch.int8, device="cuda", generator=g)
    sk = (torch.rand((1, H, N), device="cuda", generator=g) + 0.5) * 0.01
    sv = torch.full((1, H), 0.01, device="cuda")
    for Nq in (1, 400):                                  # the kernel for 32 rows, tiles of 128
        q8 = torch.randint(-127, 128, (1, H, Nq, d), dtype=torch.int8, device="cuda", generator=g)
        sq = (torch.rand((1, H, Nq), device="cuda", generator=g) + 0.5) * 3e-3
        got = ifa.int_flash_attn_fwd_window(q8, k8, k8, sq, sk, 100, s_V=sv)
        own = {"q8": q8[:, -1:], "sq": sq[:, -1:], "k8": k8[:, -1:, N - 600:], "sk": sk[:, -1:, N - 600:], "v": k8[:, -1:, N - 600:], "sv": sv[:, -1:]}
        want, tol = ref.attention({k: x.cpu() for k, x in own.items()}, torch.float16, None, 100)
        assert bool(((got[:, -1:].cpu().double() - want).abs() <= tol).all())
    q8, sq = q8[:, :, :1].contiguous(), sq[:, :, :1].contiguous()
    W = ifa.key_weights(q8, k8, sq, sk)
    alone = ifa.key_weights(q8[:, -1:].contiguous(), k8[:, -1:], sq[:, -1:].contiguous(), sk[:, -1:].contiguous())
    # each is off by less than 2 (8 max |S| 2^-24 + 2^-22) + 2^-22 + 2^-19 of itself (see cache_reference), max |S| < 40: 4.1e-5
    assert bool(((W[:, -1:] - alone).abs() <= 1e-4 * alone).all()) and abs(W[:, -1].double().sum().item() - 1) < 1e-4
    out = ifa.evict_keys(k8, sk, k8, W, 500, 20, 4)
    index = out[4][0, -1].long()
    assert torch.equal(out[0][0, -1], k8[0, -1, index]) and torch.equal(out[2][0, -1], k8[0, -1, index]) and torch.equal(out[1][0, -1], sk[0, -1, index])
    assert index[:4].tolist() == [0, 1, 2, 3] and index[-1].item() == N - 1 and bool((index[1:] > index[:-1]).all())
    assert torch.equal(index[4:-20], W[0, -1, 4:N - 20].topk(476).indices.sort().values + 4)
