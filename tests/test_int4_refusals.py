"""What int_flash_attn_fwd_int4 refuses, on the host, before anything is enqueued (no GPU)."""
import ctypes

import pytest
import torch

import paper_2409_16997_amd as ifa

P, ODD, NULL, WS = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1008), ctypes.c_void_p(0), ctypes.c_void_p(0x10000)


@pytest.fixture(scope="module")
def L():
    return ifa.lib()


def int4(L, q=P, k=P, v=P, sq=P, sk=P, sv=P, lens=NULL, B=1, H=4, Hkv=2, Nq=1, Nk=100, d=128, w=10, sinks=2, o=P, dt=1, ws=NULL, n=0):
    return L.int_flash_attn_fwd_int4(q, k, v, sq, sk, sv, lens, B, H, Hkv, Nq, Nk, d, w, sinks, o, dt, ws, n, None)


def test_int4(L):
    for name in ("q", "k", "v", "sq", "sk", "sv", "o"):
        assert int4(L, **{name: NULL}) == -1, name
    for bad in (dict(B=0), dict(H=0), dict(Hkv=0), dict(H=5), dict(Nq=0), dict(Nk=0), dict(d=0), dict(w=0), dict(w=-1), dict(sinks=-1), dict(B=1 << 30, Nk=1 << 20)):
        assert int4(L, **bad) == -2, bad
    assert int4(L, dt=3) == -3 and int4(L, dt=-1) == -3
    for bad in (dict(d=96), dict(d=32), dict(d=256), dict(Nk=0x7ff00000 // 256 + 1), dict(q=ODD), dict(k=ODD), dict(v=ODD), dict(o=ODD), dict(sq=ctypes.c_void_p(0x1002)), dict(sv=ctypes.c_void_p(0x1001)),
                dict(lens=ctypes.c_void_p(0x1002)), dict(B=1 << 22, Nk=1), dict(Nq=1 << 25, Nk=1)):
        assert int4(L, **bad) == -4, bad


def test_workspace(L):
    bytes_of = L.ifa_int4_workspace_bytes
    for shape, lens in (((1, 4, 2, 1, 8192, 128, 8192, 2), NULL), ((64, 8, 2, 1, 8192, 64, 8192, 0), P)):
        B, H, Hkv, Nq, Nk, d, w, sinks = shape
        need = bytes_of(*shape)
        assert need > 0
        big = dict(B=B, H=H, Hkv=Hkv, Nq=Nq, Nk=Nk, d=d, w=w, sinks=sinks, lens=lens)
        assert int4(L, **big) == -1
        assert int4(L, **big, ws=WS, n=0) == -6 and int4(L, **big, ws=ODD, n=need) == -4
    assert int4(L, **big, ws=WS, n=need - 1) == -6
    assert bytes_of(1, 4, 2, 1, 100, 128, 10, 2) == 0
    for bad in ((1, 4, 3, 1, 100, 128, 10, 2), (1, 4, 2, 1, 100, 128, 0, 2), (1, 4, 2, 1, 100, 100, 10, 2), (1, 4, 2, 1, 100, 128, 10, -1), (0, 4, 2, 1, 100, 128, 10, 2)):
        assert bytes_of(*bad) == -1, bad
    assert ifa.int4_workspace_bytes(1, 4, 2, 1, 8192, 128) == bytes_of(1, 4, 2, 1, 8192, 128, 8192, 0) == ifa.int4_workspace_bytes(1, 4, 2, 1, 8192, 128, 1 << 40)


def test_the_binding_names_the_operand(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    q, k, s = torch.zeros(1, 4, 1, 64, dtype=torch.int8), torch.zeros(1, 2, 9, 32, dtype=torch.uint8), torch.ones(1, 2, 9)
    with pytest.raises(ifa.IntfaError, match="Q_i8: expected a contiguous tensor in GPU memory"):
        ifa.int_flash_attn_fwd_int4(q, k, k, torch.ones(1, 4, 1), s, s)
    for bad in (torch.zeros(1, 3, 9, 32, dtype=torch.uint8), k[:, :, :0], torch.zeros(1, 2, 9, 64, dtype=torch.uint8), torch.zeros(2, 2, 9, 32, dtype=torch.uint8)):
        with pytest.raises(ifa.IntfaError, match="do not agree"):
            ifa.int_flash_attn_fwd_int4(q, bad, k, torch.ones(1, 4, 1), s, s)
    with pytest.raises(ifa.IntfaError, match="4-dimensional"):
        ifa.int_flash_attn_fwd_int4(q, k[0], k, torch.ones(1, 4, 1), s, s)
