"""Attention over a quantized cache (sliding window with sinks, shared prefix) against its definition in 64 bits."""
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


def window(ifa, s, w, sinks, lens=None, **kw):
    t = ref.on_gpu(s)
    return ifa.int_flash_attn_fwd_window(t["q8"], t["k8"], t["v"], t["sq"], t["sk"], w, sinks, s_V=t["sv"], lens=dev_lens(lens), **kw)


def prefix(ifa, s, lens=None, **kw):
    t = ref.on_gpu(s)
    return ifa.int_flash_attn_fwd_prefix(t["q8"], t["kp8"], t["vp"], t["k8"], t["v"], t["sq"], t["skp"], t["sk"], s_Vp=t["svp"], s_V=t["sv"], lens=dev_lens(lens), **kw)


def check(got, want, tol):
    got = got.cpu().double()
    off = (got - want).abs()
    assert bool((off <= tol).all()), f"off by up to {(off / tol.clamp_min(1e-300)).max().item():.3f} of the tolerance"


# B, Hkv, G, Nq, Nk, d, window, sinks, lens
WINDOWS = [
    (1, 1, 1, 1, 1, 64, 1, 0, None),                     # one key
    (2, 3, 1, 1, 33, 128, 5, 0, None),
    (2, 2, 4, 1, 300, 128, 64, 4, (300, 257)),           # a decode step, grouped heads
    (1, 1, 8, 1, 5000, 128, 4096, 4, None),              # shared out over workgroups
    (3, 2, 2, 1, 2500, 64, 2000, 100, (2500, 0, 1)),     # an empty sequence, one of one key
    (1, 2, 3, 5, 700, 128, 100, 7, (650,)),              # draft tokens, an odd group
    (1, 1, 7, 9, 1200, 64, 1000, 64, (1199,)),
    (2, 1, 1, 40, 40, 128, 3, 2, (40, 17)),              # a prompt, padded in front
    (1, 2, 1, 129, 129, 64, 1, 0, None),                 # every query sees itself alone
    (1, 1, 2, 130, 257, 128, 64, 64, None),              # a chunk; sinks as many as the window
    (1, 1, 4, 200, 200, 64, 500, 3, None),               # a window beyond the sequence: causal attention
    (2, 1, 1, 31, 95, 128, 32, 300, (95, 20)),           # more sinks than keys: causal attention
    (1, 3, 1, 300, 300, 128, 129, 1, (290,)),
    (4, 1, 1, 2, 4, 64, 2, 1, (4, 3, 2, 1)),
    (1, 1, 1, 700, 700, 128, 256, 4, None),
    (2, 8, 2, 200, 500, 64, 64, 100, (500, 333)),        # tiles of 128 rows: the seam between sinks and window inside a block, behind one, ...
    (1, 16, 3, 170, 333, 128, 70, 64, (331,)),           # ... at its end
    (3, 4, 4, 130, 130, 128, 40, 3, (130, 0, 77)),       # padded in front
    (1, 12, 1, 400, 650, 64, 1, 1, None),
    (2, 6, 4, 129, 700, 128, 10 ** 6, 0, (700, 650)),
    (9, 1, 5, 3, 64, 64, 7, 1, (64, 0, 1, 2, 3, 4, 31, 32, 33)),
]


@pytest.mark.parametrize("v,out", [("fp16", torch.float32), ("int8", torch.float16), ("fp16", torch.bfloat16)])
@pytest.mark.parametrize("case", WINDOWS, ids=[f"{i}" for i in range(len(WINDOWS))])
def test_window(ifa, case, v, out):
    B, Hkv, G, Nq, Nk, d, w, sinks, lens = case
    s = ref.problem(7, B, Hkv, G, Nq, Nk, d, v=v)
    want, tol = ref.attention(s, out, lens, w, sinks)
    check(window(ifa, s, w, sinks, lens, out_dtype=out), want, tol)


# B, Hkv, G, Nq, Np, Nk, d, lens
PREFIXES = [
    (1, 1, 1, 1, 1, 1, 64, None),
    (2, 2, 1, 1, 300, 40, 64, None),
    (3, 1, 4, 1, 33, 65, 128, (65, 0, 1)),               # nothing of its own, one key of its own
    (5, 2, 3, 2, 700, 100, 128, (100, 1, 99, 33, 0)),    # an odd group; a query in front of its own keys
    (40, 1, 4, 1, 2000, 200, 64, None),                  # more rows than a tile
    (1, 1, 8, 1, 5000, 3000, 128, (2999,)),
    (2, 1, 2, 70, 500, 300, 128, (300, 50)),             # more queries than own keys
    (7, 1, 1, 3, 32, 32, 64, (0, 1, 2, 3, 4, 31, 32)),
    (33, 2, 1, 1, 1500, 9, 128, None),
    (4, 4, 4, 80, 600, 300, 64, (300, 0, 81, 200)),      # prompts behind a prefix: tiles of 128 rows for both
    (3, 8, 2, 100, 70, 100, 128, (100, 99, 1)),
    (2, 4, 3, 200, 1500, 70, 64, (0, 69)),               # ... the keys of both in parts
    (9, 8, 2, 20, 7000, 30, 64, None),                   # ... the shared ones for the whole batch
]


@pytest.mark.parametrize("v,out", [("fp16", torch.float32), ("int8", torch.float16), ("int8", torch.bfloat16)])
@pytest.mark.parametrize("case", PREFIXES, ids=[f"{i}" for i in range(len(PREFIXES))])
def test_prefix(ifa, case, v, out):
    B, Hkv, G, Nq, Np, Nk, d, lens = case
    s = ref.problem(8, B, Hkv, G, Nq, Nk, d, Np=Np, v=v)
    want, tol = ref.attention(s, out, lens)
    check(prefix(ifa, s, lens, out_dtype=out), want, tol)


def test_what_no_query_sees_is_not_looked_at(ifa):
    """Decode steps: NaN and infinities behind L_b and in front of the window, in V and in the scales of K."""
    for d, G, L, w, sinks in ((128, 4, 900, 200, 5), (64, 1, 40, 7, 0), (128, 1, 3000, 1111, 33)):
        Nk = L + 50
        s = ref.problem(3, 1, 2, G, 1, Nk, d)
        clean, tol = ref.attention(s, torch.float16, (L,), w, sinks)
        hidden = torch.ones(Nk, dtype=torch.bool)
        hidden[:sinks] = False
        hidden[L - w:L] = False
        for bad in (math.nan, math.inf, -65504.0):
            s["v"][:, :, hidden] = bad
            s["sk"][:, :, hidden] = bad
            check(window(ifa, s, w, sinks, (L,)), clean, tol)


def test_what_no_query_of_a_prompt_sees_is_not_looked_at(ifa):
    """Chunks of a prompt (tiles of 128 rows): the same in front of the first query's window."""
    s = ref.problem(3, 1, 16, 2, 160, 900, 64)
    clean, tol = ref.attention(s, torch.float16, (880,), 100, 70)
    hidden = torch.ones(900, dtype=torch.bool)
    hidden[:70] = False
    hidden[880 - 160 - 99:880] = False
    for bad in (math.nan, math.inf):
        s["v"][:, :, hidden] = bad
        s["sk"][:, :, hidden] = bad
        check(window(ifa, s, 100, 70, (880,)), clean, tol)


@pytest.mark.parametrize("Hkv,Nq", [(1, 9), (16, 200)])       # the kernel for 32 rows, tiles of 128
def test_what_padding_queries_hold_does_not_matter(ifa, Hkv, Nq):
    s = ref.problem(2, 2, Hkv, 2, Nq, 260, 64)
    lens = (5, 0)
    want, tol = ref.attention(s, torch.float16, lens, 40, 2)
    for bad in (0.0, math.nan, math.inf):
        s["sq"][0, :, :Nq - 5] = bad
        s["sq"][1] = bad
        got = window(ifa, s, 40, 2, lens)
        check(got, want, tol)
        assert bool((got[0, :, :Nq - 5] == 0).all()) and bool((got[1] == 0).all())


def test_lengths_outside_the_buffer_count_as_the_nearer_end(ifa):
    s = ref.problem(4, 3, 1, 2, 2, 50, 64)
    a, b = window(ifa, s, 20, 2, (50, 0, 17)), window(ifa, s, 20, 2, (10 ** 9, -5, 17))
    assert torch.equal(a, b) and bool((a[1] == 0).all())


def test_out_workspace_and_stream(ifa):
    s = ref.problem(5, 1, 1, 4, 1, 6000, 128)
    t = ref.on_gpu(s)
    need = ifa.window_workspace_bytes(1, 4, 1, 1, 6000, 128, 5000, 4)
    assert need > 0
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    out = torch.full((3, 1, 4, 1, 128), 7.0, dtype=torch.float32, device="cuda")
    want = window(ifa, s, 5000, 4, out_dtype=torch.float32)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = ifa.int_flash_attn_fwd_window(t["q8"], t["k8"], t["v"], t["sq"], t["sk"], 5000, 4, out=out[1], workspace=ws)
    side.synchronize()
    assert got.data_ptr() == out[1].data_ptr() and torch.equal(out[1], want) and bool((out[0] == 7).all()) and bool((out[2] == 7).all())


def test_graph_replays(ifa):
    """Both calls in one captured graph, inputs changed between replays; every replay against the eager call."""
    s, lens = ref.problem(6, 3, 2, 4, 1, 1500, 128, Np=2500), (1500, 3, 700)
    t, ln = ref.on_gpu(s), dev_lens(lens)

    def both():
        return (ifa.int_flash_attn_fwd_window(t["q8"], t["k8"], t["v"], t["sq"], t["sk"], 1000, 4, lens=ln),
                ifa.int_flash_attn_fwd_prefix(t["q8"], t["kp8"], t["vp"], t["k8"], t["v"], t["sq"], t["skp"], t["sk"], lens=ln))

    both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = both()
    for k in range(3):
        t["q8"].copy_(torch.roll(t["q8"], 1, -1))
        ln.copy_(torch.tensor([1500 - 7 * k, 3 + k, 0], dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        eager = both()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(captured, eager))


def test_a_prefix_of_one_sequence_is_plain_attention(ifa):
    """Shared keys in front of own ones are the same keys in one buffer; a window beyond it hides nothing."""
    s = ref.problem(9, 1, 2, 2, 6, 200, 64, Np=320)
    whole = {"q8": s["q8"], "sq": s["sq"], "k8": torch.cat([s["kp8"][None], s["k8"]], 2), "sk": torch.cat([s["skp"][None], s["sk"]], 2),
             "v": torch.cat([s["vp"][None], s["v"]], 2), "sv": None}
    want, tol = ref.attention(whole, torch.float32, None, 10 ** 6)
    check(prefix(ifa, s, out_dtype=torch.float32), want, tol)
    check(window(ifa, whole, 10 ** 6, 0, out_dtype=torch.float32), want, tol)


def test_calls_on_two_streams_at_once(ifa):
    """Each call allocates a workspace of its own: calls that run side by side do not meet."""
    s = [ref.on_gpu(ref.problem(20 + k, 4, 2, 4, 1, 3000, 128, Np=4000)) for k in range(2)]

    def call(t):
        return (ifa.int_flash_attn_fwd_window(t["q8"], t["k8"], t["v"], t["sq"], t["sk"], 2000, 4), ifa.key_weights(t["q8"], t["k8"], t["sq"], t["sk"]),
                ifa.int_flash_attn_fwd_prefix(t["q8"], t["kp8"], t["vp"], t["k8"], t["v"], t["sq"], t["skp"], t["sk"]))

    want = [call(t) for t in s]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in s], []
    for _ in range(5):
        for t, stream in zip(s, streams):
            with torch.cuda.stream(stream):
                got.append(call(t))
    torch.cuda.synchronize()
    for i, g in enumerate(got):
        assert all(torch.equal(a, b) for a, b in zip(g, want[i % 2]))


def test_refusals_of_the_binding(ifa):
    t = ref.on_gpu(ref.problem(30, 2, 2, 2, 1, 3000, 64, Np=700))
    q, k, v, sq, sk = t["q8"], t["k8"], t["v"], t["sq"], t["sk"]
    lens = torch.tensor([5, 6], dtype=torch.int32, device="cuda")
    win, pre = ifa.int_flash_attn_fwd_window, ifa.int_flash_attn_fwd_prefix

    def refused(match, f, *a, **kw):
        with pytest.raises(ifa.IntfaError, match=match):
            f(*a, **kw)

    refused("window is at least 1", win, q, k, v, sq, sk, 0)
    refused("sinks at least 0", win, q, k, v, sq, sk, 4, -1)
    refused("lens", win, q, k, v, sq, sk, 4, lens=lens.long())
    refused("lens", win, q, k, v, sq, sk, 4, lens=lens[:1])
    refused("lens", win, q, k, v, sq, sk, 4, lens=lens.cpu())
    refused("V", win, q, k, v.float(), sq, sk, 4)
    refused("V", win, q, k, v, sq, sk, 4, s_V=torch.ones(2, 2, device="cuda"))
    refused("s_V", win, q, k, k, sq, sk, 4, s_V=torch.ones(2, device="cuda"))
    refused("s_Q", win, q, k, v, sq[:, :2], sk, 4)
    refused("do not agree", win, q, k.transpose(1, 2), v, sq, sk, 4)
    refused("K_i8: expected a contiguous", win, q, torch.cat([k, k], -1)[..., ::2], v, sq, sk, 4)
    refused("out", win, q, k, v, sq, sk, 4, out=torch.empty(2, 4, 1, 32, dtype=torch.float16, device="cuda"))
    refused("unsupported dtype|out_dtype|dtype", win, q, k, v, sq, sk, 4, out_dtype=torch.int32)
    refused("IFA_ERR_WORKSPACE", win, q, k, v, sq, sk, 2999, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))
    refused("uint8", win, q, k, v, sq, sk, 2999, workspace=torch.empty(1 << 22, dtype=torch.float32, device="cuda"))
    refused("both .int8 V. or neither", pre, q, t["kp8"], t["vp"], k, v, sq, t["skp"], sk, s_Vp=torch.ones(2, device="cuda"))
    refused("Vp", pre, q, t["kp8"], t["vp"][:, 1:], k, v, sq, t["skp"], sk)
    refused("at least one key", pre, q, t["kp8"][:, :0], t["vp"][:, :0], k, v, sq, t["skp"][:, :0], sk)
    refused("W", ifa.key_weights, q, k, sq, sk, W=torch.zeros(2, 2, 2999, device="cuda"))
    W = torch.zeros(2 * 2 * 3000 + 4, device="cuda")
    refused("IFA_ERR_UNSUPPORTED", ifa.key_weights, q, k, sq, sk, W=W[:-4].view(2, 2, 3000), out=W[4:].view(2, 2, 3000))
    W = W[4:].view(2, 2, 3000)
    refused("1 <= keep", ifa.evict_keys, k, sk, v, W, 3001)
    refused("1 <= keep", ifa.evict_keys, k, sk, v, W, 10, recent=8, sinks=3)
    refused("V", ifa.evict_keys, k, sk, v.bfloat16(), W, 10)
    refused("out", ifa.evict_keys, k, sk, v, W, 10, out=(k,))
    d32 = torch.zeros(1, 1, 1, 32, dtype=torch.int8, device="cuda")
    refused("not supported", win, d32, d32, d32.half(), torch.ones(1, 1, 1, device="cuda"), torch.ones(1, 1, 1, device="cuda"), 4)
