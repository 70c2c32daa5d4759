"""The operators on a quantized cache in 64 bits on the CPU, from their definitions, with how far a kernel may be off.

Where the tolerances come from (`attention`): with p_j the softmax weights of a row, O = sum p_j v_j.
  weights   each is rounded to fp16, relatively by at most 2^-11 (half a step), below 2^-14 absolutely by at most 2^-25; so is every summand of l, which the
            largest weight makes at least 1.  Numerator sum p_j |v_j| (2^-11 + ...), denominator |O| (2^-11 + ...).
  scores    int32 is exact; s_K, s_Q log2(e) and the subtraction of m round to fp32, 2^-24 each, relative to numbers of at most 2 max |S| log2(e): an absolute
            error of a score below 8 max |S| 2^-24, the same relative error of a weight.  exp2 itself: 2^-22.
  sums      fp32 additions, and parts joined with fp32 factors: n 2^-24 for n keys at the very worst; 2^-19 covers rounding errors of n = 10^4 that add up like a random walk.
  output    half a step of its type: 2^-24 relative for fp32, 2^-11 for fp16 (2^-25 absolute below its normal range), 2^-8 for bf16.
"""
import math

import torch

HALF_STEP = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}


def problem(seed, B, Hkv, G, Nq, Nk, d, Np=0, v="fp16", sigma=2.0):
    """Random operands on the CPU: codes over the whole range, scores of standard deviation about `sigma`."""
    g = torch.Generator().manual_seed(seed)

    def codes(*shape):
        return torch.randint(-127, 128, shape, generator=g).to(torch.int8)

    base = math.sqrt(sigma / (73.3 * 73.3 * math.sqrt(d)))

    def scales(*shape):
        return (torch.rand(shape, generator=g) + 0.5) * base

    def values(shape, scale_shape):
        if v == "fp16":
            return torch.randn(shape, generator=g).half(), None
        return codes(*shape), torch.rand(scale_shape, generator=g) * 0.015 + 0.005

    s = {"q8": codes(B, Hkv * G, Nq, d), "sq": scales(B, Hkv * G, Nq), "k8": codes(B, Hkv, Nk, d), "sk": scales(B, Hkv, Nk)}
    s["v"], s["sv"] = values((B, Hkv, Nk, d), (B, Hkv))
    if Np:
        s["kp8"], s["skp"] = codes(Hkv, Np, d), scales(Hkv, Np)
        s["vp"], s["svp"] = values((Hkv, Np, d), (Hkv,))
    return s


def scores(s, b, h, lens, window=None, sinks=0):
    """[Nq, Np + L_b] scores of one head in 64 bits, -inf where a query does not look."""
    q8, k8 = s["q8"], s["k8"]
    G, Nq, Nk = q8.shape[1] // k8.shape[1], q8.shape[2], k8.shape[2]
    L = Nk if lens is None else max(0, min(int(lens[b]), Nk))
    hk = h // G

    def product(k, sk):
        return (q8[b, h].double() @ k.double().T) * s["sq"][b, h].double()[:, None] * sk.double()[None]

    S = product(k8[b, hk, :L], s["sk"][b, hk, :L])
    p, j = (L - Nq + torch.arange(Nq))[:, None], torch.arange(L)[None]
    seen = j <= p
    if window is not None:
        seen = seen & ((j > p - window) | (j < sinks))
    S = S.masked_fill(~seen, -math.inf)
    if "kp8" in s:
        S = torch.cat([product(s["kp8"][hk], s["skp"][hk]), S], 1)
    return S, L


def softmax(S):
    m = S.amax(1, keepdim=True) if S.shape[1] else torch.full((S.shape[0], 1), -math.inf, dtype=torch.float64)
    e = torch.exp(S - torch.where(m.isinf(), 0.0, m))
    l = e.sum(1, keepdim=True)
    return e / torch.where(l == 0, 1.0, l)


def attention(s, out_dtype, lens=None, window=None, sinks=0):
    """(O, the most that an output may be off) as float64 [B, H, Nq, d]."""
    B, H, Nq, d = s["q8"].shape
    G = H // s["k8"].shape[1]
    O, tol = torch.zeros(B, H, Nq, d, dtype=torch.float64), torch.zeros(B, H, Nq, d, dtype=torch.float64)
    for b in range(B):
        for h in range(H):
            S, L = scores(s, b, h, lens, window, sinks)
            v = s["v"][b, h // G, :L].double() * (1.0 if s["sv"] is None else s["sv"][b, h // G].double())
            if "kp8" in s:
                v = torch.cat([s["vp"][h // G].double() * (1.0 if s["svp"] is None else s["svp"][h // G].double()), v])
            P = softmax(S)
            finite = S[~S.isinf()]
            far = 8 * (finite.abs().max().item() if finite.numel() else 0.0) * 2.0 ** -24
            rel = 2.0 ** -11 + far + 2.0 ** -22 + 2.0 ** -19
            seen = (~S.isinf()).double()
            o = P @ v
            O[b, h] = o
            tol[b, h] = rel * (P @ v.abs() + o.abs()) + 2.0 ** -25 * (seen @ v.abs() + seen.sum(1, keepdim=True) * o.abs())
    tol = tol + HALF_STEP[out_dtype] * (O.abs() + tol)
    return O, tol + (2.0 ** -25 if out_dtype == torch.float16 else 0.0)


def on_gpu(s):
    return {k: None if x is None else x.cuda() for k, x in s.items()}


def key_weights(s, lens=None, W=None):
    """(W_out, the most that an output may be off).  A weight is off relatively by what a score is (8 max |S| 2^-24) and exp2 and 1 / l are (2^-22 each), its l by the
    same and by the rounding of the sum (2^-19, as above); the sum over the rows rounds at each of its n additions by 2^-24 of at most itself."""
    B, H, Nq, _ = s["q8"].shape
    Hkv, Nk = s["k8"].shape[1:3]
    G = H // Hkv
    out, tol = torch.zeros(B, Hkv, Nk, dtype=torch.float64), torch.zeros(B, Hkv, Nk, dtype=torch.float64)
    for b in range(B):
        for h in range(H):
            S, L = scores(s, b, h, lens)
            P = softmax(S)
            finite = S[~S.isinf()]
            rel = 2 * (8 * (finite.abs().max().item() if finite.numel() else 0.0) * 2.0 ** -24 + 2.0 ** -22) + 2.0 ** -22 + 2.0 ** -19
            out[b, h // G, :L] += P.sum(0)
            tol[b, h // G, :L] += rel * P.sum(0)
    if W is not None:
        out += W.double()
    return out, tol + (G * Nq + 2) * 2.0 ** -24 * out.abs() + 1e-35


def evict(s, W, keep, recent, sinks, lens=None):
    """The six outputs, exactly."""
    B, Hkv, Nk, d = s["k8"].shape
    index = torch.full((B, Hkv, keep), -1, dtype=torch.int32)
    n_of = [Nk if lens is None else max(0, min(int(lens[b]), Nk)) for b in range(B)]
    for b, n in enumerate(n_of):
        for h in range(Hkv):
            if n <= keep:
                stay = list(range(n))
            else:
                w = W[b, h].tolist()
                middle = sorted(range(sinks, n - recent), key=lambda j: (w[j] != w[j], -w[j] if w[j] == w[j] else 0.0, j))
                stay = list(range(sinks)) + sorted(middle[:keep - sinks - recent]) + list(range(n - recent, n))
            index[b, h, :len(stay)] = torch.tensor(stay, dtype=torch.int32)
    at, there = index.clamp_min(0).long(), index >= 0

    def pick(x):
        i = at if x.dim() == 3 else at.unsqueeze(-1).expand(B, Hkv, keep, d)
        y = x.gather(2, i)
        return torch.where(there if x.dim() == 3 else there.unsqueeze(-1), y, torch.zeros_like(y))
    return pick(s["k8"]), pick(s["sk"]), pick(s["v"]), pick(W), index, torch.tensor([min(n, keep) for n in n_of], dtype=torch.int32)
