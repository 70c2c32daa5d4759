"""Attention over a cache in 4 bits in 64 bits, with the tolerance that include/intfa.h gives for V's scales row by row: what a query does not see does not count in it, and scales below 2^-80 count as that in
the tolerance, not in the value.

Where the tolerance comes from, for a row with softmax weights P, scales s_j, codes v_j (half steps throughout):
  weights   P_j s_j to fp16: 2^-11 of itself, or 2^-40 (tiles 2^-32) of max P max(|s_j|, 2^-80) over the keys that the row sees, for each |v_j| that counts
  scores    as in int4_reference.py, 8 max |S| 2^-24 + 2^-19; log2 |s_V| of up to 80 joins the exponent: its own rounding (one step of numbers below 128, 2^-17), the sum's and the difference's (half a step,
            2^-18 each) make 2^-16 of log2, less than that of the weight
  sums      2^-19 each for O and l, exp2 2^-22
  output    half a step of fp32
"""
import math

import torch

from int4_reference import unpack


def attention(s, lens=None, window=None, sinks=0, tiles=False):
    """(O, the most that an fp32 output may be off) as float64 [B, H, Nq, d]."""
    B, H, Nq, d = s["q8"].shape
    Hkv, Nk = s["k4"].shape[1:3]
    O, tol = torch.zeros(B, H, Nq, d, dtype=torch.float64), torch.zeros(B, H, Nq, d, dtype=torch.float64)
    for b in range(B):
        L = Nk if lens is None else max(0, min(int(lens[b]), Nk))
        if not L:
            continue
        p, j = (L - Nq + torch.arange(Nq))[:, None], torch.arange(L)[None]
        seen = j <= p
        if window is not None:
            seen = seen & ((j > p - window) | (j < sinks))
        for hk in range(Hkv):
            k, v = unpack(s["k4"][b, hk, :L]).double(), unpack(s["v4"][b, hk, :L]).double()
            sk, sv = s["sk"][b, hk, :L].double(), s["sv"][b, hk, :L].double()
            largest = torch.where(seen, sv.abs(), 0.0).amax(1, keepdim=True).clamp_min(2.0 ** -80)
            for h in range(hk * (H // Hkv), (hk + 1) * (H // Hkv)):
                S = ((s["q8"][b, h].double() @ k.T) * s["sq"][b, h].double()[:, None] * sk[None]).masked_fill(~seen, -math.inf)
                top = S.amax(1, keepdim=True)
                e = torch.exp(S - torch.where(top.isinf(), 0.0, top))
                l = e.sum(1, keepdim=True)
                P = e / torch.where(l == 0, 1.0, l)
                finite = S[~S.isinf()]
                rel = 8 * (finite.abs().max().item() if finite.numel() else 0.0) * 2.0 ** -24 + 2.0 ** -19 + 2.0 ** -16 + 2.0 ** -22 + 2 * 2.0 ** -19
                O[b, h] = (P * sv) @ v
                tol[b, h] = (2.0 ** -11 + rel) * ((P * sv.abs()) @ v.abs()) + rel * O[b, h].abs() + 2.0 ** (-32 if tiles else -40) * P.amax(1, keepdim=True) * largest * (seen.double() @ v.abs())
    return O, tol + 2.0 ** -24 * (O.abs() + tol)
