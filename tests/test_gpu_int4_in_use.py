"""The calls on a cache in 4 bits together, as a program uses them: prompts and steps appended and attended to, rotated keys, graphs, streams, caches beyond 32 bits of offset."""
import math

import pytest
import torch

import append_reference as written
import int4_reference as ref

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


def empty(B, Hkv, Nk, d):
    return [x.cuda() for x in written.empty_cache("i4", B, Hkv, Nk, d)]


@pytest.mark.parametrize("B,Hkv,G,N,steps,Nk,d", [(2, 2, 2, 150, 6, 160, 64), (3, 4, 4, 400, 4, 900, 128), (64, 2, 1, 30, 3, 3600, 64), (2, 40, 1, 640, 2, 1000, 64)])
def test_prompts_and_steps(ifa, B, Hkv, G, N, steps, Nk, d):
    """Ragged prompts padded in front, rotated keys, then single tokens; the cache against its definition, each output against the cache."""
    g = torch.Generator().manual_seed(Nk)
    lens = torch.tensor([max(0, N - 17 * b) for b in range(B)], dtype=torch.int32)
    ln, cache = lens.cuda(), empty(B, Hkv, Nk, d)
    host = written.empty_cache("i4", B, Hkv, Nk, d)
    for step in range(1 + steps):
        n = 1 if step else N
        q = (torch.randn(B, Hkv * G, n, d, generator=g) * 2).half()
        k, v = ((torch.randn(B, n, Hkv, d, generator=g) * 2).bfloat16().transpose(1, 2) for _ in range(2))      # as a projection leaves them
        if step:
            lens += 1
            ln += 1
        q8, sq = ifa.quantize_tokenwise(q.cuda(), scale_mul=d ** -0.5 / d, hadamard=True)
        ifa.append_keys(k.cuda(), v.cuda(), *cache, lens=ln, hadamard=True)
        O = ifa.int_flash_attn_fwd_int4(q8, cache[0], cache[2], sq, cache[1], cache[3], lens=ln)
        host = written.append("i4", k, v, host, lens, True)
        for a, b in zip(cache, host):
            assert torch.equal(a.cpu(), b)
        s = {"q8": q8.cpu(), "sq": sq.cpu(), "k4": host[0], "sk": host[1], "v4": host[2], "sv": host[3]}
        close(O, *ref.attention(s, torch.float16, lens))
        back = ifa.read_keys(*cache, lens=ln, first=None, count=n, hadamard=True, out_dtype=torch.bfloat16)
        for a, b in zip(back, written.read("i4", host, lens, None, n, True, torch.bfloat16)):
            assert torch.equal(a.cpu(), b)


def test_what_four_bits_cost(ifa):
    """Against attention to the unquantized values: the error that steps of a / 7 have, with loud channels only when K is rotated."""
    B, Hkv, G, N, d = 1, 2, 4, 600, 128
    g = torch.Generator().manual_seed(0)
    loud = torch.ones(d)
    loud[:4] = 20.0
    q, k, v = torch.randn(B, Hkv * G, 8, d, generator=g) / loud, torch.randn(B, Hkv, N, d, generator=g) * loud, torch.randn(B, Hkv, N, d, generator=g)
    S = (q.double() @ k.double().repeat_interleave(G, 1).transpose(-1, -2)) * d ** -0.5
    S = S.masked_fill(torch.arange(N) > N - 8 + torch.arange(8)[:, None], -math.inf)
    want = torch.softmax(S, -1) @ v.double().repeat_interleave(G, 1)
    off = {}
    for rotated in (False, True):
        cache = empty(B, Hkv, N, d)
        ifa.append_keys(k.cuda(), v.cuda(), *cache, hadamard=rotated)
        q8, sq = ifa.quantize_tokenwise(q.cuda(), scale_mul=d ** -0.5 / (d if rotated else 1), hadamard=rotated)
        O = ifa.int_flash_attn_fwd_int4(q8, cache[0], cache[2], sq, cache[1], cache[3])
        off[rotated] = ((O.cpu().double() - want).norm() / want.norm()).item()
    # A step of a / 7, a = 2.7 rms of the row on average, leaves errors of .111 rms.  V's are .111 of its values, which the weights average alike: .111 of O.  Scores: the rows of K have a norm of
    # sqrt(124 + 4 x 400) = 41.5, rotated their channels have 41.5 rms (unnormalized) and errors of 4.6; a score sums them weighed by the rotated q, whose norm is sqrt(128) sqrt(124) = 126, times
    # 1 / (128 sqrt(128)): errors of 126 x 4.6 / 1448 = .40, as much of each weight.  Together sqrt(.40^2 + .111^2) = .415; a quarter more for what a is in 600 rows of 2 heads.
    # Not rotated the step is 20 x 2 / 7 = 5.7 for channels of 1, which all become 0, and with them the scores but for what the loud channels give.
    assert off[True] < 0.52, off
    assert off[False] > 1.5 * off[True], off


def capture(fn):
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        fn()
        fn()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fn()
    return graph


@pytest.mark.parametrize("B,Hkv,G,Nk,d", [(2, 2, 2, 300, 64), (2, 2, 4, 3000, 128), (64, 2, 2, 3400, 64)])
def test_a_captured_step_replays_to_the_eager_result(ifa, B, Hkv, G, Nk, d):
    """append, attention and read in one graph, the lengths counted up inside it; eager work on other tensors between the replays."""
    g = torch.Generator(device="cuda").manual_seed(1)
    r = lambda *s: torch.randn(s, device="cuda", generator=g)  # noqa: E731
    first = torch.tensor([Nk // 2 - 3 * b for b in range(B)], dtype=torch.int32, device="cuda").clamp_min(0)
    start = empty(B, Hkv, Nk, d)
    ifa.append_keys(r(B, Hkv, Nk, d).half(), r(B, Hkv, Nk, d).half(), *start)
    need = ifa.int4_workspace_bytes(B, Hkv * G, Hkv, 1, Nk, d)

    def program():
        s = {"q": r(B, Hkv * G, 1, d).half(), "k": r(B, Hkv, 1, d).half(), "v": r(B, Hkv, 1, d).half(), "lens": first.clone(), "cache": [x.clone() for x in start],
             "O": torch.empty(B, Hkv * G, 1, d, dtype=torch.float16, device="cuda"), "back": tuple(torch.empty(B, Hkv, 1, d, dtype=torch.float16, device="cuda") for _ in range(2)),
             "ws": torch.empty(max(need, 1), dtype=torch.uint8, device="cuda")}

        def step():
            s["lens"] += 1
            ifa.append_keys(s["k"], s["v"], *s["cache"], lens=s["lens"])
            q8, sq = ifa.quantize_tokenwise(s["q"], scale_mul=d ** -0.5)
            c = s["cache"]
            ifa.int_flash_attn_fwd_int4(q8, c[0], c[2], sq, c[1], c[3], lens=s["lens"], out=s["O"], workspace=s["ws"])
            ifa.read_keys(*c, lens=s["lens"], first=None, count=1, out=s["back"])
        return s, step

    (replayed, step), (eager, eager_step) = program(), program()
    graph = capture(step)
    replayed["lens"].copy_(first)
    for x, y in zip(replayed["cache"], start):
        x.copy_(y)
    for _ in range(5):
        q, k, v = r(B, Hkv * G, 1, d).half(), r(B, Hkv, 1, d).half(), r(B, Hkv, 1, d).half()
        for s in (replayed, eager):
            s["q"].copy_(q), s["k"].copy_(k), s["v"].copy_(v)
        graph.replay()
        eager_step()
        torch.cuda.synchronize()
        assert torch.equal(replayed["O"], eager["O"]) and torch.equal(replayed["lens"], eager["lens"])
        assert all(torch.equal(a, b) for a, b in zip(replayed["cache"] + list(replayed["back"]), eager["cache"] + list(eager["back"])))
        r(100, 100) @ r(100, 100)


def test_calls_side_by_side(ifa):
    """Two streams with calls of their own, eagerly and as two graphs that replay at once; the current stream is the one that a call goes to."""
    calls = []
    for seed, shape in ((1, (2, 2, 4, 2, 3000, 128)), (2, (64, 2, 2, 1, 3400, 64))):
        B, Hkv, G, Nq, Nk, d = shape
        t = ref.on_gpu(ref.problem(seed, *shape))
        ln = torch.tensor([Nk - 7 * b for b in range(B)], dtype=torch.int32, device="cuda")
        calls.append(lambda t=t, ln=ln: ifa.int_flash_attn_fwd_int4(t["q8"], t["k4"], t["v4"], t["sq"], t["sk"], t["sv"], lens=ln))
    want = [c() for c in calls]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        got = []
        for s, c in zip(streams, calls):
            with torch.cuda.stream(s):
                got.append([c() for _ in range(3)])
        torch.cuda.synchronize()
        assert all(torch.equal(x, w) for xs, w in zip(got, want) for x in xs)
    out = [None, None]

    def record(i):
        out[i] = calls[i]()
    graphs = [capture(lambda i=i: record(i)) for i in range(2)]
    for _ in range(5):
        for s, graph in zip(streams, graphs):
            with torch.cuda.stream(s):
                graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))
        for x in out:
            x.zero_()
        torch.cuda.synchronize()


@pytest.mark.parametrize("Nq,window", [(1, 300), (128, 4000)])
def test_offsets_beyond_32_bits(ifa, Nq, window):
    """70 heads of 2^20 keys: 4.7 GB of codes each for K and V; the last keys of the last heads."""
    B, Hkv, Nk, d, tail = 1, 70, 1 << 20, 128, 5000
    g = torch.Generator().manual_seed(3)
    cache = [torch.zeros(B, Hkv, Nk, d // 2, dtype=torch.uint8, device="cuda"), torch.zeros(B, Hkv, Nk, device="cuda"), torch.zeros(B, Hkv, Nk, d // 2, dtype=torch.uint8, device="cuda"),
             torch.zeros(B, Hkv, Nk, device="cuda")]
    K, V = (torch.randn(B, Hkv, tail, d, generator=g).half() for _ in range(2))
    ifa.append_keys(K.cuda(), V.cuda(), *cache)
    host = written.append("i4", K, V, written.empty_cache("i4", B, Hkv, tail, d), None, False)
    assert all(torch.equal(x[:, :, -tail:].cpu(), y) for x, y in zip(cache, host))
    assert not cache[0][:, :, :-tail].any() and not cache[3][:, :, :-tail].any()
    back = ifa.read_keys(*cache, first=Nk - 100, count=100)
    assert all(torch.equal(x.cpu(), y) for x, y in zip(back, written.read("i4", host, None, tail - 100, 100, False, torch.float16)))
    q8, sq = ifa.quantize_tokenwise(torch.randn(B, Hkv, Nq, d, generator=g).cuda(), scale_mul=d ** -0.5)
    O = ifa.int_flash_attn_fwd_int4(q8, cache[0], cache[2], sq, cache[1], cache[3], window=window)
    s = {"q8": q8[:, -2:].cpu(), "sq": sq[:, -2:].cpu(), "k4": host[0][:, -2:], "sk": host[1][:, -2:], "v4": host[2][:, -2:], "sv": host[3][:, -2:]}
    close(O[:, -2:], *ref.attention(s, torch.float16, None, window))
