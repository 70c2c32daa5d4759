"""A cache that is quantized as it is written, as cases that can be timed: what a layer does with the keys and values of new
tokens, and attention over a cache held in 4 bits.

  append   K and V of new tokens quantized into their slots of the cache, and what the cache now holds for them read back
           (so that a prompt can go on with the values that later steps will see)
  read     a run of the cache given back as values
  int4     attention of queries to a cache held in 4 bits: a prompt, draft tokens, a decode step

The cache is held in one of three ways ("held"):
  i8f16    K in INT8 with a scale per token and head, V in fp16
  i8       V in INT8, too, with one scale per head that the program has from a calibration
  i4       K and V in 4 bits, -7 .. 7 with a scale per token and head; byte j of a row holds channel j in its low four bits
           and channel j + d/2 in its high ones, both as code + 8
"rotated": K goes through the Walsh-Hadamard transform before it is quantized, and back when it is read.

Sequence b has L_b keys in buffers of Nk ("lens": all of them, or lengths from none to all of them), new ones included: the
Nn new tokens, and the Nq queries, are its last positions, token i at p = L_b - Nn + i.  One at p < 0 is padding: it is not
written, reads as zeros, and as a query gives zeros.  A query at p sees keys j <= p with j > p - window or j < sinks.
Hq = G Hkv query heads share Hkv key heads; Q is INT8 with a scale per token (the softmax scale is part of it).
"""
import math

import torch

own = False

DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}
LARGEST = {"i8f16": 127.0, "i8": 127.0, "i4": 7.0}


def _append(name, B, Hkv, Nn, Nk, d, held, x="fp16", tokens_first=False, lens="full", rotated=False):
    c = {"op": "append", "B": B, "Hkv": Hkv, "Nn": Nn, "Nk": Nk, "d": d, "held": held, "x": x, "tokens_first": tokens_first,
         "lens": lens, "rotated": rotated}
    return dict(c, name=name) if name else c


def _read(name, B, Hkv, first, count, Nk, d, held, x="fp16", lens="full", rotated=False):
    c = {"op": "read", "B": B, "Hkv": Hkv, "first": first, "count": count, "Nk": Nk, "d": d, "held": held, "x": x, "lens": lens,
         "rotated": rotated}
    return dict(c, name=name) if name else c


def _int4(name, B, Hkv, G, Nq, Nk, d, window=0, sinks=0, lens="full", out="fp16"):
    """window 0: every key up to the query's own."""
    c = {"op": "int4", "B": B, "Hkv": Hkv, "G": G, "Nq": Nq, "Nk": Nk, "d": d, "window": window, "sinks": sinks, "lens": lens,
         "out": out}
    return dict(c, name=name) if name else c


def listed():
    return [
        # a prompt of a batch goes into the cache, K and V as the projection leaves them, token by token
        _append("append_prompt_8192", 4, 8, 8192, 8192, 128, "i4", "bf16", True),
        # a decode step's new token of many requests
        _append("append_decode_64", 64, 8, 1, 4096, 128, "i4", "fp16", True, "ragged"),
        # ragged prompts, padded in front, small heads, from fp32, rotated, V by a calibrated scale
        _append("append_ragged_1777", 3, 12, 1777, 2048, 64, "i8", "fp32", False, "ragged", True),
        # the smallest calls: one short sequence's new token, where latency counts
        _append("append_one", 1, 4, 1, 700, 64, "i8f16"),
        # the whole cache of a batch given back, for a kernel that wants values
        _read("read_batch_16", 16, 8, 0, 16384, 16384, 128, "i4", "bf16", "ragged"),
        # a piece of a short one, rotated back
        _read("read_piece_260", 2, 8, 40, 260, 340, 64, "i8", "fp32", "full", True),
        # a decode step of a batch deep inside its sequences
        _int4("int4_decode_16", 16, 8, 4, 1, 16384, 128, lens="ragged"),
        # a decode step of one very long sequence
        _int4("int4_decode_131072", 1, 8, 4, 1, 131072, 128),
        # the smallest: one short sequence's decode step
        _int4("int4_decode_one", 1, 4, 2, 1, 700, 64),
        # draft tokens of a few requests, large groups, bf16 out
        _int4("int4_draft_8x5", 8, 4, 8, 5, 16391, 128, lens="ragged", out="bf16"),
        # prompts of two requests, grouped heads: the largest call
        _int4("int4_prompt_4096", 2, 8, 4, 4096, 4096, 128),
        # ragged prompts, padded in front, with a window and a sink, small heads, bf16 out
        _int4("int4_window_1777", 3, 12, 1, 1777, 1777, 64, 333, 1, "ragged", "bf16"),
    ]


def _log(rng, lo, hi):
    """An integer between lo and hi, even over the logarithm."""
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


MOST_SCORES = 2 * 32 * 4096 * 4096 // 2     # of int4_prompt_4096: half of its square
MOST_CACHE = 16 * 8 * 16384 * 128           # elements of K, of the largest cache
MOST_NEW = 4 * 8 * 8192 * 128               # of K of append_prompt_8192


def draw(rng):
    """Another case of the same ranges: 1 to 64 sequences of up to 131072 keys, both head sizes, any group of heads."""
    while True:
        op = rng.choice(["append", "append", "read", "int4", "int4", "int4"])
        d, lens, x = rng.choice([64, 128, 128]), rng.choice(["full", "ragged"]), rng.choice(["fp16", "bf16", "fp32"])
        Hkv, held, rotated = rng.choice([1, 2, 4, 8, 8, 12, 32]), rng.choice(["i4", "i4", "i8", "i8f16"]), rng.random() < 0.3
        B, Nk = _log(rng, 1, 64), _log(rng, 64, 131072)
        few = rng.choice([1, 1, rng.randint(2, 8), rng.randint(9, 40)])
        if op == "append":
            Nn = min(Nk, few if rng.random() < 0.5 else _log(rng, 16, 8192))
            c = _append(None, B, Hkv, Nn, Nk, d, held, x, rng.random() < 0.5, lens, rotated)
            if B * Hkv * Nn * d > MOST_NEW:
                continue
        elif op == "read":
            first = rng.choice([0, 0, rng.randint(0, Nk - 1)])
            c = _read(None, B, Hkv, first, rng.choice([Nk - first, rng.randint(1, Nk - first)]), Nk, d, held, x, lens, rotated)
        else:
            G, Nq = rng.choice([1, 1, 2, 3, 4, 4, 7, 8]), min(Nk, few if rng.random() < 0.6 else _log(rng, 32, 8192))
            window, sinks = rng.choice([(0, 0), (0, 0), (_log(rng, 16, 8192), rng.choice([0, 1, 4, 100]))])
            c = _int4(None, B, Hkv, G, Nq, Nk, d, window, sinks, lens, rng.choice(["fp16", "bf16"]))
            if B * Hkv * G * Nq * Nk > MOST_SCORES:
                continue
        if B * Hkv * Nk * d <= MOST_CACHE:
            return c


def _lens(case):
    """L_b: full buffers, or lengths spread from none to all of the buffer (a lone sequence: two thirds of it)."""
    B, Nk = case["B"], case["Nk"]
    if case["lens"] == "full":
        return [Nk] * B
    return [Nk - Nk // 3] if B == 1 else [Nk * b // (B - 1) for b in range(B)]


def _pack(q):
    """Codes -7 .. 7 as bytes: channel j and, above it, channel j + d/2."""
    u = (q + 8.0).to(torch.uint8)
    h = u.shape[-1] // 2
    return u[..., :h] | (u[..., h:] << 4)


def _unpack(w):
    return torch.cat([w & 15, w >> 4], -1).float() - 8.0


def _quantize(x, largest):
    """(codes as fp32 numbers, scales) of rows: the largest magnitude becomes `largest`."""
    a = x.abs().amax(-1, keepdim=True)
    some, most = a > 0, torch.full_like(a, largest)
    inv = torch.where(some, most / a, torch.zeros_like(a))
    return torch.round(x * inv).clamp_(-largest, largest), torch.where(some, a / most, torch.ones_like(a)).squeeze(-1)


def _rotate(x):
    """The Walsh-Hadamard transform of every row (Sylvester order, unnormalized), butterflies of 1, 2, 4, ... apart."""
    d, h = x.shape[-1], 1
    while h < d:
        y = x.view(*x.shape[:-1], d // (2 * h), 2, h)
        x = torch.stack([y[..., 0, :] + y[..., 1, :], y[..., 0, :] - y[..., 1, :]], -2).flatten(-3)
        h *= 2
    return x


def _held(held, k, v, sv=None):
    """K and V (fp32) as the cache holds them: (K, s_K, V, s_V)."""
    qk, sk = _quantize(k, LARGEST[held])
    if held == "i4":
        qv, sv = _quantize(v, 7.0)
        return _pack(qk), sk, _pack(qv), sv
    if held == "i8f16":
        return qk.to(torch.int8), sk, v.half(), None
    inv = torch.where(sv != 0, 1.0 / sv, torch.zeros_like(sv))
    return qk.to(torch.int8), sk, torch.round(v * inv[..., None, None]).clamp_(-127, 127).to(torch.int8), sv


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    op, B, Hkv, Nk, d = (case[k] for k in ("op", "B", "Hkv", "Nk", "d"))
    held = case.get("held", "i4")
    n = lambda *shape: torch.randn(shape, device="cuda", generator=g)  # noqa: E731
    s = {"case": case, "lens": None if case["lens"] == "full" else torch.tensor(_lens(case), dtype=torch.int32, device="cuda")}
    direction = n(d)
    loud = 1.0 + 4.0 * (torch.rand(d, device="cuda", generator=g) < 0.03)      # a few channels of K are several times the others

    def keys(*lead):                       # a few directions that many queries look for, the first keys among what they find
        k = n(*lead, d)
        hit = torch.rand(lead, device="cuda", generator=g) < 0.01
        hit[..., :2] = True
        return (k + hit[..., None] * (1.5 * direction)) * loud

    def values(*lead):                     # tokens differ in how much they say
        return n(*lead, d) * torch.exp(0.3 * n(*lead, 1))

    sv = torch.rand((B, Hkv), device="cuda", generator=g) * 0.01 + 0.03 if held == "i8" else None
    if op == "append":
        s["cache"] = _held(held, torch.zeros(B, Hkv, Nk, d, device="cuda"), torch.zeros(B, Hkv, Nk, d, device="cuda"), sv)
        lead = (B, case["Nn"], Hkv) if case["tokens_first"] else (B, Hkv, case["Nn"])
        s["k"], s["v"] = keys(*lead).to(DTYPES[case["x"]]), values(*lead).to(DTYPES[case["x"]])
        if case["tokens_first"]:
            s["k"], s["v"] = s["k"].transpose(1, 2), s["v"].transpose(1, 2)
        return s
    k = keys(B, Hkv, Nk)
    s["cache"] = _held(held, _rotate(k) if case.get("rotated") else k, values(B, Hkv, Nk), sv)
    if op == "int4":
        q, sq = _quantize((1.5 * n(B, Hkv * case["G"], case["Nq"], d) + 0.5 * direction) / loud, 127.0)
        s["q8"], s["sq"] = q.to(torch.int8), sq * d ** -0.5
    return s


def _L(s):
    case = s["case"]
    return s["lens"].long().view(-1, 1, 1) if s["lens"] is not None else torch.full((case["B"], 1, 1), case["Nk"], device="cuda")


def _values(case, cache, there):
    """What the rows of a cache stand for, zeros where `there` is false."""
    kc, sk, vc, sv = cache
    if case["held"] == "i4":
        k, v = _unpack(kc), _unpack(vc) * sv.unsqueeze(-1)
    elif case["held"] == "i8":
        k, v = kc.float(), vc.float() * sv[..., None, None]
    else:
        k, v = kc.float(), vc.float()
    k = k * sk.unsqueeze(-1)
    if case["rotated"]:
        k = _rotate(k) / case["d"]
    x = DTYPES[case["x"]]
    there = there.unsqueeze(-1)
    return torch.where(there, k, 0.0).to(x), torch.where(there, v, 0.0).to(x)


def _plain_append(s):
    case = s["case"]
    B, Hkv, Nn, Nk = (case[k] for k in ("B", "Hkv", "Nn", "Nk"))
    k, v = s["k"].float(), s["v"].float()
    kc, sk, vc, sv = s["cache"]
    new = _held(case["held"], _rotate(k) if case["rotated"] else k, v, sv)
    p = _L(s) - Nn + torch.arange(Nn, device="cuda")
    there = (p >= 0).expand(B, Hkv, Nn)
    at = (torch.arange(B, device="cuda").view(B, 1, 1), torch.arange(Hkv, device="cuda").view(1, Hkv, 1), p % Nk)    # padding: a slot behind the last key, as it was
    for to, rows in zip((kc, sk, vc, sv if case["held"] == "i4" else None), new):
        if to is not None:
            to[at] = torch.where(there.unsqueeze(-1) if to.dim() == 4 else there, rows, to[at])
    back = (kc[at], sk[at], vc[at], sv[at] if case["held"] == "i4" else sv)
    k, v = _values(case, back, there)
    return {"k": k, "v": v, "sk": sk, "sv": sv if case["held"] == "i4" else None}


def _plain_read(s):
    case = s["case"]
    a, b = case["first"], case["first"] + case["count"]
    kc, sk, vc, sv = s["cache"]
    there = (torch.arange(a, b, device="cuda") < _L(s)).expand(case["B"], case["Hkv"], case["count"])
    k, v = _values(case, (kc[:, :, a:b], sk[:, :, a:b], vc[:, :, a:b], sv[:, :, a:b] if case["held"] == "i4" else sv), there)
    return {"k": k, "v": v}


def _plain_int4(s):
    case = s["case"]
    B, Hkv, G, Nq, Nk, d = (case[k] for k in ("B", "Hkv", "G", "Nq", "Nk", "d"))
    kc, sk, vc, sv = s["cache"]
    S = s["q8"].view(B, Hkv, G * Nq, d).float() @ _unpack(kc).transpose(-1, -2)
    S = S.mul_(s["sq"].view(B, Hkv, G * Nq, 1)).mul_(sk.unsqueeze(-2)).view(B, Hkv, G, Nq, Nk)
    p = (_L(s) - Nq + torch.arange(Nq, device="cuda").view(1, 1, Nq)).view(B, Nq, 1)
    j = torch.arange(Nk, device="cuda")
    seen = j <= p
    if case["window"]:
        seen &= (j > p - case["window"]) | (j < case["sinks"])
    S = S.masked_fill_(~seen.view(B, 1, 1, Nq, Nk), -math.inf)
    m = S.amax(-1, keepdim=True)
    P = S.sub_(torch.where(m == -math.inf, torch.zeros_like(m), m)).exp_()
    l = P.sum(-1, keepdim=True)
    O = P.view(B, Hkv, G * Nq, Nk) @ (_unpack(vc) * sv.unsqueeze(-1))
    return O.div_(torch.where(l == 0, torch.ones_like(l), l).view(B, Hkv, G * Nq, 1)).view(B, Hkv * G, Nq, d).to(DTYPES[case["out"]])


def _own(s):
    import paper_2409_16997_amd as ifa
    case = s["case"]
    kc, sk, vc, sv = s["cache"]
    if case["op"] == "int4":
        return ifa.int_flash_attn_fwd_int4(s["q8"], kc, vc, s["sq"], sk, sv, window=case["window"] or None, sinks=case["sinks"], lens=s["lens"],
                                           out_dtype=DTYPES[case["out"]])
    x = DTYPES[case["x"]]
    if case["op"] == "read":
        k, v = ifa.read_keys(kc, sk, vc, sv, lens=s["lens"], first=case["first"], count=case["count"], hadamard=case["rotated"], out_dtype=x)
        return {"k": k, "v": v}
    ifa.append_keys(s["k"], s["v"], kc, sk, vc, sv, lens=s["lens"], hadamard=case["rotated"])
    k, v = ifa.read_keys(kc, sk, vc, sv, lens=s["lens"], first=None, count=case["Nn"], hadamard=case["rotated"], out_dtype=x)     # the last Nn
    return {"k": k, "v": v, "sk": sk, "sv": sv if case["held"] == "i4" else None}


def run(s):
    if own:
        return _own(s)
    return {"append": _plain_append, "read": _plain_read, "int4": _plain_int4}[s["case"]["op"]](s)


def _row_bytes(case):
    """Bytes of a key and its value, scales included, in the cache."""
    d, held = case["d"], case.get("held", "i4")
    return {"i4": d + 8, "i8": 2 * d + 4, "i8f16": 3 * d + 4}[held]


def work(case):
    op, B, Hkv, Nk, d = (case[k] for k in ("op", "B", "Hkv", "Nk", "d"))
    lens = _lens(case)
    x = {"fp16": 2, "bf16": 2, "fp32": 4}.get(case.get("x"))
    if op == "append":                     # the tokens in, into the cache, and what they are there out
        rows = Hkv * sum(min(n, case["Nn"]) for n in lens)
        return {"bytes": rows * (2 * d * x + _row_bytes(case)) + Hkv * B * case["Nn"] * 2 * d * x, "flops": 0.0}
    if op == "read":
        a, b = case["first"], case["first"] + case["count"]
        return {"bytes": Hkv * (sum(max(0, min(n, b) - a) for n in lens) * _row_bytes(case) + B * case["count"] * 2 * d * x), "flops": 0.0}
    G, Nq, window, sinks = case["G"], case["Nq"], case["window"] or Nk, case["sinks"]
    pairs, keys = 0, 0
    for n in lens:
        p = torch.arange(max(n - Nq, 0), n)                      # positions of the queries that see anything
        if not len(p):
            continue
        lo = (p - window + 1).clamp_min(0)
        pairs += int((p + 1 - lo + lo.clamp_max(sinks)).sum())
        keys += n - int(lo[0]) + min(int(lo[0]), sinks)
    rows = B * Hkv * G * Nq
    return {"bytes": rows * (d + 4 + 2 * d) + Hkv * keys * _row_bytes(case), "flops": 4.0 * Hkv * G * pairs * d}


def _exact_rotation(x):
    """Channel j after a step is x[j] + x[j + h] where bit h of j is 0 and x[j - h] - x[j] where it is 1, rounded to 32 bits by the
    definition (next to a border that decides the code)."""
    j = torch.arange(x.shape[-1], device=x.device)
    for e in range(x.shape[-1].bit_length() - 1):
        x = (x[..., j & ~(1 << e)] + x[..., j | (1 << e)] * (1.0 - 2.0 * (j >> e & 1))).float().double()
    return x


def _exact_codes(x, largest):
    """Codes by the definition, whose product is rounded to 32 bits (what it is next to a border decides), and scales in 64."""
    a = x.abs().amax(-1, keepdim=True)
    inv = (largest / torch.where(a == 0, math.inf, a)).float().double()
    return (x * inv).float().double().round().clamp(-largest, largest), torch.where(a == 0, 1.0, a / largest)


def exact(case, seed):
    s = prepare(case, seed)
    op, B, Hkv, Nk, d = (case[k] for k in ("op", "B", "Hkv", "Nk", "d"))
    lens = _lens(case)
    if op == "int4":
        return _exact_int4(s, lens)
    H = torch.ones(1, 1, dtype=torch.float64, device="cuda")
    while H.shape[0] < d:
        H = torch.cat([torch.cat([H, H], 1), torch.cat([H, -H], 1)])
    held, rotated = case["held"], case["rotated"]
    kc, sk, vc, sv = s["cache"]

    def nibbles(w):
        return torch.cat([w.long() % 16, w.long() // 16], -1).double() - 8.0

    if op == "read":
        k, v = [], []
        for b, n in enumerate(lens):
            at = torch.arange(case["first"], case["first"] + case["count"], device="cuda")
            keep = (at < n).double()[:, None]
            kk = (nibbles(kc[b][:, at]) if held == "i4" else kc[b][:, at].double()) * sk[b][:, at, None].double()
            k.append((kk @ H / d if rotated else kk) * keep)
            vv = nibbles(vc[b][:, at]) * sv[b][:, at, None].double() if held == "i4" else vc[b][:, at].double()
            v.append((vv * sv[b, :, None, None].double() if held == "i8" else vv) * keep)
        return {"k": torch.stack(k), "v": torch.stack(v)}
    Nn = case["Nn"]
    k, v = torch.zeros(B, Hkv, Nn, d, dtype=torch.float64, device="cuda"), torch.zeros(B, Hkv, Nn, d, dtype=torch.float64, device="cuda")
    scale_k, scale_v = sk.double(), sv.double() if held == "i4" else None
    for b, n in enumerate(lens):
        new = min(n, Nn)
        if not new:
            continue
        x, y = s["k"][b, :, Nn - new:].double(), s["v"][b, :, Nn - new:].double()
        q, a = _exact_codes(_exact_rotation(x) if rotated else x, LARGEST[held])
        k[b, :, Nn - new:] = q * a @ H / d if rotated else q * a
        scale_k[b, :, n - new:n] = a[..., 0]
        if held == "i4":
            q, a = _exact_codes(y, 7.0)
            y = q * a
            scale_v[b, :, n - new:n] = a[..., 0]
        elif held == "i8":
            t = sv[b].double()[:, None, None]
            y = (y * (1.0 / t).float().double()).float().double().round().clamp(-127, 127) * t
        else:
            y = y.half().double()
        v[b, :, Nn - new:] = y
    return {"k": k, "v": v, "sk": scale_k, "sv": scale_v}


def _exact_int4(s, lens):
    case = s["case"]
    B, Hkv, G, Nq, Nk, d = (case[k] for k in ("B", "Hkv", "G", "Nq", "Nk", "d"))
    window, sinks = case["window"] or Nk, case["sinks"]
    kc, sk, vc, sv = s["cache"]
    out = torch.zeros(B, Hkv * G, Nq, d, dtype=torch.float64, device="cuda")
    step = max(1, (1 << 27) // Nk)
    for b, n in enumerate(lens):
        first = max(0, Nq - n)                                   # the queries before it see nothing
        for hk in range(Hkv):
            k, v = (torch.cat([w.long() % 16, w.long() // 16], -1).double() - 8.0 for w in (kc[b, hk, :n], vc[b, hk, :n]))
            k, v = k * sk[b, hk, :n, None].double(), v * sv[b, hk, :n, None].double()
            for h in range(hk * G, hk * G + G):
                for i0 in range(first, Nq, step):
                    i = torch.arange(i0, min(Nq, i0 + step), device="cuda")
                    S = (s["q8"][b, h, i].double() * s["sq"][b, h, i, None].double()) @ k.T
                    p, j = (n - Nq + i)[:, None], torch.arange(n, device="cuda")[None]
                    S[(j > p) | ((p - j >= window) & (j >= sinks))] = -math.inf
                    out[b, h, i] = torch.softmax(S, 1) @ v
    return out
