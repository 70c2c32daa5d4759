"""Attention over a cache in 4 bits in 64 bits on the CPU, from its definition, with how far a kernel may be off.

Where the tolerance comes from: with P the softmax of a row, s_j the scale of V's token j, v_j its codes, O = sum P_j s_j v_j.
  weights   P_j s_j is rounded to fp16, relatively by at most 2^-11 (half a step), below fp16's normal range absolutely by at most 2^-25 of its unit.  The unit is 2^-7 at most (tiles; the
            kernel for few rows 2^-15) of a bound of P_j s_j that is no more than the largest P times the largest |s|: 2^-32 of that product, for each |v_j| that counts.
  scores    int32 is exact; s_K, s_Q log2(e) and the subtraction of M round to fp32, 2^-24 each, relative to numbers of at most 2 max |S| log2(e) plus the distance of M, below 2^5 here: an
            absolute error of a score below 8 max |S| 2^-24 + 2^-19, the same relative error of a weight.  exp2 itself: 2^-22.
  sums      fp32 additions, parts joined with fp32 factors: 2^-19, as rounding errors of n = 10^4 summands add up like a random walk.
  output    half a step of its type.
"""
import math

import torch

HALF_STEP = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}


def unpack(w):
    return torch.cat([(w & 15).to(torch.int8), (w >> 4).to(torch.int8)], -1) - 8


def problem(seed, B, Hkv, G, Nq, Nk, d, sigma=2.0):
    """Random operands on the CPU: every code there is, scores of standard deviation about `sigma`."""
    g = torch.Generator().manual_seed(seed)

    def nibbles():
        return torch.randint(0, 256, (B, Hkv, Nk, d // 2), generator=g).to(torch.uint8)

    base = math.sqrt(sigma / (73.3 * 4.6 * math.sqrt(d)))
    return {"q8": torch.randint(-127, 128, (B, Hkv * G, Nq, d), generator=g).to(torch.int8), "sq": (torch.rand(B, Hkv * G, Nq, generator=g) + 0.5) * base,
            "k4": nibbles(), "sk": (torch.rand(B, Hkv, Nk, generator=g) + 0.5) * base, "v4": nibbles(), "sv": torch.exp(0.5 * torch.randn(B, Hkv, Nk, generator=g)) * 0.2}


def attention(s, out_dtype, lens=None, window=None, sinks=0):
    """(O, the most that an output may be off) as float64 [B, H, Nq, d]."""
    B, H, Nq, d = s["q8"].shape
    Hkv, Nk = s["k4"].shape[1:3]
    O, tol = torch.zeros(B, H, Nq, d, dtype=torch.float64), torch.zeros(B, H, Nq, d, dtype=torch.float64)
    for b in range(B):
        L = Nk if lens is None else max(0, min(int(lens[b]), Nk))
        p, j = (L - Nq + torch.arange(Nq))[:, None], torch.arange(L)[None]
        seen = j <= p
        if window is not None:
            seen = seen & ((j > p - window) | (j < sinks))
        for hk in range(Hkv):
            k, v = unpack(s["k4"][b, hk, :L]).double(), unpack(s["v4"][b, hk, :L]).double()
            sk, sv = s["sk"][b, hk, :L].double(), s["sv"][b, hk, :L].double()
            for h in range(hk * (H // Hkv), (hk + 1) * (H // Hkv)):
                if not L:
                    continue
                S = ((s["q8"][b, h].double() @ k.T) * s["sq"][b, h].double()[:, None] * sk[None]).masked_fill(~seen, -math.inf)
                top = S.amax(1, keepdim=True)
                e = torch.exp(S - torch.where(top.isinf(), 0.0, top))
                l = e.sum(1, keepdim=True)
                P = e / torch.where(l == 0, 1.0, l)
                finite = S[~S.isinf()]
                rel = 8 * (finite.abs().max().item() if finite.numel() else 0.0) * 2.0 ** -24 + 2.0 ** -19 + 2.0 ** -22 + 2.0 ** -19
                o = (P * sv) @ v
                O[b, h] = o
                Ps = P * sv.abs()
                tol[b, h] = (2.0 ** -11 + rel) * (Ps @ v.abs()) + rel * o.abs() + 2.0 ** -32 * P.amax(1, keepdim=True) * sv.abs().max() * (seen.double() @ v.abs())
    tol = tol + HALF_STEP[out_dtype] * (O.abs() + tol)
    return O, tol + (2.0 ** -25 if out_dtype == torch.float16 else 0.0)


def on_gpu(s):
    return {k: x.cuda() for k, x in s.items()}
