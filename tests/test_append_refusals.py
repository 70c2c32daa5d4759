"""What append_keys and read_keys refuse, on the host, before anything is enqueued (no GPU)."""
import ctypes

import pytest
import torch

import paper_2409_16997_amd as ifa

I8_F16, I8, I4 = 0, 1, 2
BASE = [(1 + i) << 32 for i in range(8)]


@pytest.fixture(scope="module")
def L():
    return ifa.lib()


def append(L, at=BASE, dt=1, ks=(0, 0, 0), vs=(0, 0, 0), B=2, Hkv=3, Nn=5, Nk=100, d=128, held=I4):
    """`at`: addresses of K, V, lens, K_c, s_K, V_c, s_V (0: null)."""
    k, v, lens, kc, sk, vc, sv = (ctypes.c_void_p(x) for x in at[:7])
    return L.append_keys(k, v, dt, *ks, *vs, lens, B, Hkv, Nn, Nk, d, held, 0, kc, sk, vc, sv, None)


def read(L, at=BASE, dt=1, B=2, Hkv=3, Nk=100, d=128, held=I4, first=0, count=100):
    """`at`: addresses of K_c, s_K, V_c, s_V, lens, K, V."""
    kc, sk, vc, sv, lens, k, v = (ctypes.c_void_p(x) for x in at[:7])
    return L.read_keys(kc, sk, vc, sv, lens, B, Hkv, Nk, d, held, 0, first, count, k, v, dt, None)


def put(i, x):
    return BASE[:i] + [x] + BASE[i + 1:]


def test_append(L):
    for i in (0, 1, 3, 4, 5, 6):
        assert append(L, put(i, 0)) == -1, i
    assert append(L, put(6, 0), held=I8) == -1
    for bad in (dict(B=0), dict(Hkv=0), dict(Nn=0), dict(Nn=-1), dict(Nk=0), dict(d=0), dict(ks=(-8, 0, 0)), dict(vs=(0, 0, -8)), dict(vs=(1 << 42, 0, 0)), dict(B=1 << 20, Hkv=1 << 10, Nk=1 << 20)):
        assert append(L, **bad) == -2, bad
    for bad in (dict(dt=3), dict(dt=-1), dict(held=3), dict(held=-1)):
        assert append(L, **bad) == -3, bad
    for bad in (dict(d=32), dict(d=256), dict(B=1 << 15, Hkv=1 << 10, Nn=9, Nk=64, d=64), dict(ks=(4, 0, 0)), dict(vs=(0, 0, 12)), dict(ks=(0, 2, 0), dt=0)):
        assert append(L, **bad) == -4, bad
    for i, off in ((0, 8), (1, 8), (3, 8), (5, 8), (2, 2), (4, 2), (6, 2)):
        assert append(L, put(i, BASE[i] + off)) == -4, i
    # the cache's arrays apart from the tokens, lens and each other: 2 x 3 x 100 keys of 64 bytes and a scale of 4
    for i, n in ((3, 600 * 64), (4, 2400), (5, 600 * 64), (6, 2400)):
        for j in range(7):
            if j != i:
                assert append(L, put(j, BASE[i])) == -4 and append(L, put(j, BASE[i] + n - 16)) == -4, (i, j)
    assert append(L, put(0, BASE[3] - 16)) == -4         # tokens that reach into it
    assert append(L, put(0, BASE[3] - 4096), ks=(0, 1024, 128)) == -4


def test_read(L):
    for i in (0, 1, 2, 3, 5, 6):
        assert read(L, put(i, 0)) == -1, i
    for bad in (dict(B=0), dict(Hkv=-1), dict(Nk=0), dict(d=0), dict(count=0), dict(first=-2), dict(first=101), dict(B=1 << 20, Hkv=1 << 10, Nk=1, count=1 << 20)):
        assert read(L, **bad) == -2, bad
    for bad in (dict(dt=3), dict(dt=-1), dict(held=3), dict(held=-1)):
        assert read(L, **bad) == -3, bad
    for bad in (dict(d=96), dict(B=1 << 15, Hkv=1 << 10, Nk=1, count=9)):
        assert read(L, **bad) == -4, bad
    for i, off in ((0, 8), (2, 8), (5, 8), (6, 8), (1, 2), (3, 2), (4, 2)):
        assert read(L, put(i, BASE[i] + off)) == -4, i
    for i in (5, 6):
        for j in range(7):
            if j != i:
                assert read(L, put(j, BASE[i])) == -4, (i, j)


def cache(d=64, four=True):
    if four:
        return torch.zeros(1, 2, 9, d // 2, dtype=torch.uint8), torch.ones(1, 2, 9), torch.zeros(1, 2, 9, d // 2, dtype=torch.uint8), torch.ones(1, 2, 9)
    return torch.zeros(1, 2, 9, d, dtype=torch.int8), torch.ones(1, 2, 9), torch.zeros(1, 2, 9, d).half(), None


def test_the_binding_names_the_operand(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    k = torch.zeros(1, 2, 3, 64)
    with pytest.raises(ifa.IntfaError, match="K_c: expected a contiguous tensor in GPU memory"):
        ifa.append_keys(k, k, *cache())
    with pytest.raises(ifa.IntfaError, match="K_c: expected a contiguous tensor in GPU memory"):
        ifa.read_keys(*cache(four=False))
    with pytest.raises(ifa.IntfaError, match="not empty"):
        ifa.append_keys(k, k, cache()[0][:, :0], *cache()[1:])
    with pytest.raises(ifa.IntfaError, match="not empty"):
        ifa.read_keys(None, *cache()[1:])
