"""Serving a long context from the quantized cache, as cases that can be timed: what a layer does when it does not look at
every key of every sequence each time.

  window   attention in which a query sees the last `window` keys up to its own position and the first `sinks` of the
           sequence: a prompt, a chunk of one, a decode step
  prefix   attention of a batch whose sequences begin with the same keys (one long document or instruction, many
           requests): the shared keys are held once, each sequence has its own keys behind them
  weights  the softmax weight that each key of the cache has drawn, added up over queries: what eviction goes by
  evict    the cache cut down to `keep` keys a head: the first `sinks`, the last `recent` and those of the largest weight,
           moved together in their order

K is INT8 with a scale per token, Q too (the softmax scale is part of it), and V is fp16 or INT8 with a scale per head
("v").  Hq = G Hkv query heads share Hkv key heads.  Sequence b has L_b keys in buffers of Nk ("lens": all of them, or
lengths from none to all of them); its Nq queries are its last positions, i.e. query i stands at p = L_b - Nq + i, and one
at p < 0 sees nothing and gives zeros.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}


def _window(name, B, Hkv, G, Nq, Nk, d, window, sinks, lens="full", v="fp16", out="fp16"):
    c = {"op": "window", "B": B, "Hkv": Hkv, "G": G, "Nq": Nq, "Nk": Nk, "d": d, "window": window, "sinks": sinks,
         "lens": lens, "v": v, "out": out}
    return dict(c, name=name) if name else c


def _prefix(name, B, Hkv, G, Nq, Np, Nk, d, lens="full", v="fp16", out="fp16"):
    c = {"op": "prefix", "B": B, "Hkv": Hkv, "G": G, "Nq": Nq, "Np": Np, "Nk": Nk, "d": d, "lens": lens, "v": v, "out": out}
    return dict(c, name=name) if name else c


def _weights(name, B, Hkv, G, Nq, Nk, d, lens="full", past=True):
    c = {"op": "weights", "B": B, "Hkv": Hkv, "G": G, "Nq": Nq, "Nk": Nk, "d": d, "lens": lens, "past": past}
    return dict(c, name=name) if name else c


def _evict(name, B, Hkv, Nk, d, keep, recent, sinks, lens="full", v="fp16"):
    c = {"op": "evict", "B": B, "Hkv": Hkv, "Nk": Nk, "d": d, "keep": keep, "recent": recent, "sinks": sinks, "lens": lens, "v": v}
    return dict(c, name=name) if name else c


def listed():
    return [
        # prompts of a batch, window a quarter of them, grouped heads
        _window("window_prompt_4096", 4, 8, 4, 4096, 4096, 128, 1024, 4),
        # one long prompt with a wide window, a head of keys for each head of queries: the largest call
        _window("window_prompt_8192", 1, 32, 1, 8192, 8192, 128, 4096, 16),
        # ragged prompts of a batch, padded in front, small heads, INT8 V, bf16 out
        _window("window_ragged_1777", 3, 12, 1, 1777, 1777, 64, 333, 1, "ragged", "int8", "bf16"),
        # a decode step of a batch deep inside its sequences
        _window("window_decode_16", 16, 8, 4, 1, 16384, 128, 4096, 4, "ragged"),
        # the smallest calls: one short sequence's decode step, where latency counts
        _window("window_decode_one", 1, 4, 2, 1, 700, 64, 256, 4, "full", "int8"),
        # a decode step of 64 requests on one document
        _prefix("prefix_decode_64", 64, 8, 4, 1, 8192, 512, 128, "ragged"),
        # draft tokens of a few requests on a longer one, INT8 V, bf16 out
        _prefix("prefix_draft_8x5", 8, 4, 8, 5, 16391, 1000, 128, "ragged", "int8", "bf16"),
        # two requests that share a short instruction
        _prefix("prefix_pair", 2, 8, 1, 1, 300, 40, 64),
        # what a decode step of a batch adds to the weights of its cache
        _weights("weights_decode_16", 16, 8, 4, 1, 16384, 128, "ragged"),
        # the weights of a whole prompt
        _weights("weights_prompt_4096", 1, 8, 4, 4096, 4096, 128, past=False),
        # the cache of a batch cut to a quarter
        _evict("evict_batch_16", 16, 8, 16384, 128, 4096, 512, 4),
        # a short one's, INT8 V
        _evict("evict_one", 1, 4, 700, 64, 256, 32, 4, v="int8"),
    ]


def _log(rng, lo, hi):
    """An integer between lo and hi, even over the logarithm."""
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


MOST_SCORES = 32 * 8192 * 8192      # of window_prompt_8192
MOST_CACHE = 16 * 8 * 16384 * 128   # elements of K, of the decode step of a batch


def draw(rng):
    """Another case of the same ranges: 1 to 64 sequences of up to 32768 keys, both head sizes, any group of heads."""
    while True:
        op = rng.choice(["window", "window", "prefix", "weights", "evict"])
        d, lens, v, out = rng.choice([64, 128, 128]), rng.choice(["full", "ragged"]), rng.choice(["fp16", "fp16", "int8"]), rng.choice(["fp16", "bf16"])
        Hkv, G = rng.choice([1, 2, 4, 8, 8, 12, 32]), rng.choice([1, 1, 2, 3, 4, 4, 7, 8])
        few = rng.choice([1, 1, rng.randint(2, 8), rng.randint(9, 40)])
        if op == "prefix":
            B = _log(rng, 1, 64)
            c = _prefix(None, B, Hkv, G, few, _log(rng, 64, 32768), _log(rng, 1, 2048), d, lens, v, out)
            keys, scores = Hkv * (c["Np"] + B * c["Nk"]), B * Hkv * G * few * (c["Np"] + c["Nk"])
        else:
            B, Nk = _log(rng, 1, 32), _log(rng, 64, 32768)
            Nq = few if rng.random() < 0.6 else _log(rng, 32, 8192)
            keys, scores = B * Hkv * Nk, B * Hkv * G * Nq * Nk
            if op == "window":
                c = _window(None, B, Hkv, G, min(Nq, Nk), Nk, d, _log(rng, 16, 8192), rng.choice([0, 1, 4, 4, 64, 100]), lens, v, out)
            elif op == "weights":
                c = _weights(None, B, Hkv, G, min(Nq, Nk), Nk, d, lens, rng.random() < 0.5)
            else:
                keep = _log(rng, 16, Nk)
                recent = rng.choice([0, keep // 8, keep // 2])
                c, scores = _evict(None, B, Hkv, Nk, d, keep, recent, rng.choice([0, min(4, keep - recent)]), lens, v), 0
        if keys * d <= MOST_CACHE and scores <= MOST_SCORES // 2:
            return c


def _lens(case):
    """L_b: full buffers, or lengths spread from none to all of the buffer (a lone sequence: two thirds of it)."""
    B, Nk = case["B"], case["Nk"]
    if case["lens"] == "full":
        return [Nk] * B
    return [Nk - Nk // 3] if B == 1 else [Nk * b // (B - 1) for b in range(B)]


def _codes(x, factor=1.0):
    """INT8 codes and the scale of each row, as a program's quantizer leaves them."""
    a = x.abs().amax(-1, keepdim=True).clamp_min(1e-20)
    return torch.round(x * (127.0 / a)).clamp_(-127, 127).to(torch.int8), (a[..., 0] * (factor / 127.0)).contiguous()


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    op, B, Hkv, Nk, d = (case[k] for k in ("op", "B", "Hkv", "Nk", "d"))
    n = lambda *shape: torch.randn(shape, device="cuda", generator=g)  # noqa: E731
    s = {"case": case, "lens": None if case["lens"] == "full" else torch.tensor(_lens(case), dtype=torch.int32, device="cuda")}

    def keys(*lead):                       # a few directions that many queries look for, the first keys among what they find
        k = n(*lead, d)
        hit = torch.rand(lead, device="cuda", generator=g) < 0.01
        hit[..., :2] = True
        return _codes(k + hit[..., None] * (1.5 * direction))

    def values(lead, scales):
        x = n(*lead, d)
        if case["v"] == "fp16":
            return x.half(), None
        return torch.round(x * 31.75).clamp_(-127, 127).to(torch.int8), torch.rand(scales, device="cuda", generator=g) * 0.01 + 0.03

    direction = n(d)
    s["k8"], s["sk"] = keys(B, Hkv, Nk)
    if op == "evict":
        s["v"], _ = values((B, Hkv, Nk), (B, Hkv))
        s["w"] = torch.exp(2.0 * n(B, Hkv, Nk)) * (torch.rand((B, Hkv, Nk), device="cuda", generator=g) > 0.1)    # some keys were never looked at
        return s
    s["q8"], s["sq"] = _codes(1.5 * n(B, Hkv * case["G"], case["Nq"], d) + 0.5 * direction, d ** -0.5)
    if op == "weights":
        s["w"] = torch.exp(n(B, Hkv, Nk)) * (4.0 * case["G"] * case["Nq"] / Nk) if case["past"] else None     # a few such calls' worth
        return s
    s["v"], s["sv"] = values((B, Hkv, Nk), (B, Hkv))
    if op == "prefix":
        s["kp8"], s["skp"] = keys(Hkv, case["Np"])
        s["vp"], s["svp"] = values((Hkv, case["Np"]), (Hkv,))
    return s


def _seen(s, device):
    """[B, 1, 1, Nq, Nk]: which keys a query sees."""
    case = s["case"]
    B, Nq, Nk = case["B"], case["Nq"], case["Nk"]
    L = s["lens"].long() if s["lens"] is not None else torch.full((B,), Nk, device=device)
    p = L.view(B, 1, 1) - Nq + torch.arange(Nq, device=device).view(1, Nq, 1)
    j = torch.arange(Nk, device=device).view(1, 1, Nk)
    seen = j <= p
    if case["op"] == "window":
        seen &= (j > p - case["window"]) | (j < case["sinks"])
    return seen.view(B, 1, 1, Nq, Nk)


def _scores(s):
    """[B, Hkv, G, Nq, Nk] in fp32, -inf where a query does not look."""
    case = s["case"]
    B, Hkv, G, Nq, Nk, d = (case[k] for k in ("B", "Hkv", "G", "Nq", "Nk", "d"))
    S = s["q8"].view(B, Hkv, G * Nq, d).float() @ s["k8"].float().transpose(-1, -2)
    S = S.mul_(s["sq"].view(B, Hkv, G * Nq, 1)).mul_(s["sk"].unsqueeze(-2)).view(B, Hkv, G, Nq, Nk)
    return S.masked_fill_(~_seen(s, S.device), -math.inf)


def _softmax(S):
    """exp(S - max) in place of S, and its sum; a row that sees nothing has 0 and 1."""
    m = S.amax(-1, keepdim=True)
    P = S.sub_(torch.where(m == -math.inf, torch.zeros_like(m), m)).exp_()
    l = P.sum(-1, keepdim=True)
    return P, torch.where(l == 0, torch.ones_like(l), l)


def _plain_window(s):
    case = s["case"]
    B, Hkv, G, Nq, Nk, d = (case[k] for k in ("B", "Hkv", "G", "Nq", "Nk", "d"))
    P, l = _softmax(_scores(s))
    O = (P.view(B, Hkv, G * Nq, Nk) @ s["v"].float()).div_(l.view(B, Hkv, G * Nq, 1))
    if s["sv"] is not None:
        O = O * s["sv"].view(B, Hkv, 1, 1)
    return O.view(B, Hkv * G, Nq, d).to(DTYPES[case["out"]])


def _plain_prefix(s):
    case = s["case"]
    B, Hkv, G, Nq, Np, Nk, d = (case[k] for k in ("B", "Hkv", "G", "Nq", "Np", "Nk", "d"))
    q = s["q8"].view(B, Hkv, G * Nq, d).transpose(0, 1).reshape(Hkv, B * G * Nq, d).float()    # every row of the batch against the one prefix
    Sp = (q @ s["kp8"].float().transpose(-1, -2)).view(Hkv, B, G * Nq, Np).transpose(0, 1)
    Sp = Sp * s["sq"].view(B, Hkv, G * Nq, 1) * s["skp"].view(1, Hkv, 1, Np)
    P, l = _softmax(torch.cat([Sp, _scores(s).view(B, Hkv, G * Nq, Nk)], -1))
    vp, v = s["vp"].float(), s["v"].float()
    if s["sv"] is not None:
        vp, v = vp * s["svp"].view(Hkv, 1, 1), v * s["sv"].view(B, Hkv, 1, 1)
    Pp = P[..., :Np].transpose(0, 1).reshape(Hkv, B * G * Nq, Np)
    O = (Pp @ vp).view(Hkv, B, G * Nq, d).transpose(0, 1) + P[..., Np:] @ v
    return (O / l).reshape(B, Hkv * G, Nq, d).to(DTYPES[case["out"]])


def _plain_weights(s):
    P, l = _softmax(_scores(s))
    W = P.div_(l).sum((2, 3), dtype=torch.float64)
    return (W if s["w"] is None else s["w"] + W).float()


def _plain_evict(s):
    case = s["case"]
    B, Hkv, Nk, d, keep, recent, sinks = (case[k] for k in ("B", "Hkv", "Nk", "d", "keep", "recent", "sinks"))
    L = s["lens"].view(B, 1, 1) if s["lens"] is not None else torch.full((B, 1, 1), Nk, device="cuda")
    j = torch.arange(Nk, device="cuda").view(1, 1, Nk)
    w = s["w"].masked_fill((j < sinks) | (j >= L - recent), math.inf).masked_fill(j >= L, -math.inf)
    index = w.sort(dim=-1, descending=True, stable=True).indices[..., :keep].masked_fill_(torch.arange(keep, device="cuda") >= L, Nk).sort(-1).values
    there = index < Nk
    at = index.clamp_max(Nk - 1)
    row = at.unsqueeze(-1).expand(B, Hkv, keep, d)
    return {"k8": s["k8"].gather(2, row) * there.unsqueeze(-1), "sk": s["sk"].gather(2, at) * there, "v": s["v"].gather(2, row) * there.unsqueeze(-1),
            "w": s["w"].gather(2, at) * there, "index": torch.where(there, index, -1).int(), "lens": L.view(B).clamp_max(keep).int()}


def _own(s):
    import paper_2409_16997_amd as ifa
    case = s["case"]
    op = case["op"]
    if op == "window":
        return ifa.int_flash_attn_fwd_window(s["q8"], s["k8"], s["v"], s["sq"], s["sk"], case["window"], case["sinks"], s_V=s["sv"], lens=s["lens"],
                                             out_dtype=DTYPES[case["out"]])
    if op == "prefix":
        return ifa.int_flash_attn_fwd_prefix(s["q8"], s["kp8"], s["vp"], s["k8"], s["v"], s["sq"], s["skp"], s["sk"], s_Vp=s["svp"], s_V=s["sv"], lens=s["lens"],
                                             out_dtype=DTYPES[case["out"]])
    if op == "weights":
        return ifa.key_weights(s["q8"], s["k8"], s["sq"], s["sk"], W=s["w"], lens=s["lens"])
    k8, sk, v, w, index, lens = ifa.evict_keys(s["k8"], s["sk"], s["v"], s["w"], case["keep"], case["recent"], case["sinks"], lens=s["lens"])
    return {"k8": k8, "sk": sk, "v": v, "w": w, "index": index, "lens": lens}


def run(s):
    if own:
        return _own(s)
    return {"window": _plain_window, "prefix": _plain_prefix, "weights": _plain_weights, "evict": _plain_evict}[s["case"]["op"]](s)


def work(case):
    op, B, Hkv, Nk, d = (case[k] for k in ("op", "B", "Hkv", "Nk", "d"))
    lens = _lens(case)
    v = d * (2 if case.get("v") == "fp16" else 1)
    if op == "evict":                  # every weight is looked at, the rows that stay are read and written
        rows = sum(min(n, case["keep"]) for n in lens)
        return {"bytes": Hkv * (4 * sum(lens) + 2 * rows * (d + v + 8) + 4 * B * case["keep"]), "flops": 0.0}
    G, Nq = case["G"], case["Nq"]
    heads, pairs, keys = Hkv * G, 0, 0
    for n in lens:
        p = np.arange(max(n - Nq, 0), n, dtype=np.int64)        # positions of the queries that see anything
        if not len(p):
            continue
        if op == "window":
            lo = np.maximum(p - case["window"] + 1, 0)
            pairs += int((p + 1 - lo + np.minimum(lo, case["sinks"])).sum())
            keys += n - int(lo[0]) + min(int(lo[0]), case["sinks"])
        else:
            pairs += int((p + 1).sum())
            keys += n
    q = B * heads * Nq * (d + 4)
    if op == "weights":                # K once, the weights in and out
        return {"bytes": q + Hkv * (keys * (d + 4) + 4 * B * Nk * (2 if case["past"] else 1)), "flops": 2.0 * heads * pairs * d}
    if op == "prefix":
        pairs, keys = pairs + B * Nq * case["Np"], keys + case["Np"]
    return {"bytes": q + Hkv * keys * (d + 4 + v) + B * heads * Nq * d * 2, "flops": 4.0 * heads * pairs * d}


def _exact_rows(q, sq, k, sk):
    return (q.double() @ k.double().T) * sq.double()[:, None] * sk.double()[None, :]


def exact(case, seed):
    s = prepare(case, seed)
    op, B, Hkv, Nk, d = (case[k] for k in ("op", "B", "Hkv", "Nk", "d"))
    lens = _lens(case)
    if op == "evict":
        return _exact_evict(s, lens)
    G, Nq = case["G"], case["Nq"]
    if op == "weights":
        out = torch.zeros(B, Hkv, Nk, dtype=torch.float64, device="cuda")
    else:
        out = torch.zeros(B, Hkv * G, Nq, d, dtype=torch.float64, device="cuda")
    step = max(1, (1 << 27) // Nk)
    for b, n in enumerate(lens):
        first = max(0, Nq - n)                                   # the queries before it see nothing of the sequence's own
        for h in range(Hkv * G):
            hk = h // G
            k, sk = s["k8"][b, hk, :n], s["sk"][b, hk, :n]
            for i0 in range(0, Nq, step):
                i = torch.arange(i0, min(Nq, i0 + step), device="cuda")
                S = _exact_rows(s["q8"][b, h, i], s["sq"][b, h, i], k, sk)
                p = (n - Nq + i)[:, None]
                j = torch.arange(n, device="cuda")[None]
                hidden = j > p
                if op == "window":
                    hidden |= (p - j >= case["window"]) & (j >= case["sinks"])
                S[hidden] = -math.inf
                if op == "prefix":
                    S = torch.cat([_exact_rows(s["q8"][b, h, i], s["sq"][b, h, i], s["kp8"][hk], s["skp"][hk]), S], 1)
                else:
                    S = S[i >= first]
                if not S.numel():
                    continue
                P = torch.softmax(S, 1)
                if op == "weights":
                    out[b, hk, :n] += P.sum(0)
                    continue
                v = s["v"][b, hk, :n].double() * (1.0 if s["sv"] is None else s["sv"][b, hk].double())
                if op == "prefix":
                    out[b, h, i] = P @ torch.cat([s["vp"][hk].double() * (1.0 if s["sv"] is None else s["svp"][hk].double()), v])
                else:
                    out[b, h, i[i >= first]] = P @ v
    if op == "weights" and s["w"] is not None:
        out += s["w"].double()
    return out


def _exact_evict(s, lens):
    case = s["case"]
    B, Hkv, Nk, d, keep, recent, sinks = (case[k] for k in ("B", "Hkv", "Nk", "d", "keep", "recent", "sinks"))
    w = s["w"].cpu().numpy().astype(np.float64)
    index = np.full((B, Hkv, keep), -1, np.int32)
    for b, n in enumerate(lens):
        for h in range(Hkv):
            if n <= keep:
                index[b, h, :n] = np.arange(n)
                continue
            middle = np.arange(sinks, n - recent)
            best = middle[np.lexsort((middle, -w[b, h, middle]))][:keep - sinks - recent]
            index[b, h] = np.concatenate([np.arange(sinks), np.sort(best), np.arange(n - recent, n)])
    at = torch.from_numpy(index).cuda().long()

    def rows(x):
        x = torch.cat([x, torch.zeros_like(x[:, :, :1])], 2)     # index -1: the row of zeros behind the last
        return torch.stack([torch.stack([x[b, h][at[b, h]] for h in range(Hkv)]) for b in range(B)])
    return {"k8": rows(s["k8"]), "sk": rows(s["sk"]).double(), "v": rows(s["v"]) if case["v"] == "int8" else rows(s["v"]).double(),
            "w": rows(s["w"]).double(), "index": at.int(), "lens": torch.tensor([min(n, keep) for n in lens], dtype=torch.int32)}
