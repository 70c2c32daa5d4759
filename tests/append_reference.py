"""append_keys and read_keys from their definition, on the CPU in float32 (whose single operations round once), bit for bit."""
import torch

LARGEST = {"i8f16": 127.0, "i8": 127.0, "i4": 7.0}
LEAST4 = 2.0 ** -118


def rotate(x):
    """Walsh-Hadamard, Sylvester order, unnormalized: fp32 butterflies of 1, 2, 4, ... apart."""
    d, h = x.shape[-1], 1
    while h < d:
        y = x.reshape(*x.shape[:-1], d // (2 * h), 2, h)
        x = torch.stack([y[..., 0, :] + y[..., 1, :], y[..., 0, :] - y[..., 1, :]], -2).flatten(-3)
        h *= 2
    return x


def codes(x, largest):
    """(codes, scales) of rows of fp32 numbers."""
    a = x.abs().amax(-1)
    some = a >= LEAST4 if largest == 7.0 else a > 0
    inv = torch.where(some, torch.full_like(a, largest) / torch.where(some, a, torch.ones_like(a)), torch.zeros_like(a))
    return torch.round(x * inv[..., None]).clamp(-largest, largest), torch.where(some, a / torch.full_like(a, largest), torch.ones_like(a))


def pack(q):
    u = (q + 8).to(torch.uint8)
    h = u.shape[-1] // 2
    return u[..., :h] | (u[..., h:] << 4)


def unpack(w):
    return torch.cat([w & 15, w >> 4], -1).float() - 8.0


def empty_cache(held, B, Hkv, Nk, d, sv=None):
    """A cache whose bytes say that nobody has written them."""
    if held == "i4":
        return [torch.full((B, Hkv, Nk, d // 2), 0x5a, dtype=torch.uint8), torch.full((B, Hkv, Nk), -3.0), torch.full((B, Hkv, Nk, d // 2), 0xa5, dtype=torch.uint8), torch.full((B, Hkv, Nk), -5.0)]
    v = torch.full((B, Hkv, Nk, d), 77.0).to(torch.int8 if held == "i8" else torch.float16)
    return [torch.full((B, Hkv, Nk, d), 99, dtype=torch.int8), torch.full((B, Hkv, Nk), -3.0), v, sv]


def length(lens, b, Nk):
    return Nk if lens is None else max(0, min(int(lens[b]), Nk))


def append(held, K, V, cache, lens, rotated):
    """The cache after the call (a new one)."""
    Kc, sK, Vc, sV = (None if x is None else x.clone() for x in cache)
    B, Hkv, Nn, _ = K.shape
    Nk = Kc.shape[2]
    k, v = K.float(), V.float()
    qk, sk = codes(rotate(k) if rotated else k, LARGEST[held])
    if held == "i4":
        qv, sv = codes(v, 7.0)
        nk, nv = pack(qk), pack(qv)
    else:
        nk = qk.to(torch.int8)
        if held == "i8":
            inv = torch.where(sV != 0, 1.0 / torch.where(sV != 0, sV, torch.ones_like(sV)), torch.zeros_like(sV))
            nv = torch.round(v * inv[..., None, None]).clamp(-127, 127).to(torch.int8)
        else:
            nv = v.half()
    for b in range(B):
        L = length(lens, b, Nk)
        n = min(L, Nn)
        if n:
            Kc[b, :, L - n:L], sK[b, :, L - n:L], Vc[b, :, L - n:L] = nk[b, :, Nn - n:], sk[b, :, Nn - n:], nv[b, :, Nn - n:]
            if held == "i4":
                sV[b, :, L - n:L] = sv[b, :, Nn - n:]
    return [Kc, sK, Vc, sV]


def read(held, cache, lens, first, count, rotated, dtype):
    Kc, sK, Vc, sV = cache
    B, Hkv, Nk = sK.shape
    if held == "i4":
        k, v = unpack(Kc) * sK[..., None], unpack(Vc) * sV[..., None]
    else:
        k, v = Kc.float() * sK[..., None], Vc.float() * (sV[..., None, None] if held == "i8" else 1.0)
    d = k.shape[-1]
    if rotated:
        k = rotate(k) * (1.0 / d)
    out = [torch.zeros(B, Hkv, count, d), torch.zeros(B, Hkv, count, d)]
    for b in range(B):
        L = length(lens, b, Nk)
        for i in range(count):
            p = (L - count if first is None else first) + i
            if 0 <= p < L:
                out[0][b, :, i], out[1][b, :, i] = k[b, :, p], v[b, :, p]
    return [x.to(dtype) for x in out]
