"""What the calls on a quantized cache refuse, on the host, before anything is enqueued (no GPU)."""
import ctypes

import pytest
import torch

import paper_2409_16997_amd as ifa

P, ODD, NULL, WS = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1008), ctypes.c_void_p(0), ctypes.c_void_p(0x10000)


@pytest.fixture(scope="module")
def L():
    return ifa.lib()


def window(L, q=P, k=P, v=P, sq=P, sk=P, sv=NULL, lens=NULL, B=1, H=4, Hkv=2, Nq=1, Nk=100, d=128, w=10, sinks=2, o=P, dt=1, ws=NULL, n=0):
    return L.int_flash_attn_fwd_window(q, k, v, sq, sk, sv, lens, B, H, Hkv, Nq, Nk, d, w, sinks, o, dt, ws, n, None)


def prefix(L, q=P, kp=P, vp=P, k=P, v=P, sq=P, skp=P, sk=P, svp=NULL, sv=NULL, lens=NULL, B=1, H=4, Hkv=2, Nq=1, Np=50, Nk=100, d=128, o=P, dt=1, ws=WS, n=1 << 40):
    return L.int_flash_attn_fwd_prefix(q, kp, vp, k, v, sq, skp, sk, svp, sv, lens, B, H, Hkv, Nq, Np, Nk, d, o, dt, ws, n, None)


def test_window(L):
    for name in ("q", "k", "v", "sq", "sk", "o"):
        assert window(L, **{name: NULL}) == -1, name
    for bad in (dict(B=0), dict(H=0), dict(Hkv=0), dict(H=5), dict(Nq=0), dict(Nk=0), dict(d=0), dict(w=0), dict(w=-1), dict(sinks=-1), dict(B=1 << 30, Nk=1 << 20)):
        assert window(L, **bad) == -2, bad
    assert window(L, dt=3) == -3 and window(L, dt=-1) == -3
    for bad in (dict(d=96), dict(d=32), dict(Nk=0x7ff00000 // 256 + 1), dict(q=ODD), dict(k=ODD), dict(v=ODD), dict(o=ODD), dict(sq=ctypes.c_void_p(0x1002)),
                dict(lens=ctypes.c_void_p(0x1002)), dict(B=1 << 22, Nk=1), dict(Nq=1 << 25, Nk=1)):
        assert window(L, **bad) == -4, bad
    big = dict(Nk=8192, w=8192)
    need = L.ifa_window_workspace_bytes(1, 4, 2, 1, 8192, 128, 8192, 2)
    assert need > 0
    assert window(L, **big) == -1
    assert window(L, **big, ws=WS, n=need - 1) == -6 and window(L, **big, ws=ODD, n=need) == -4
    assert L.ifa_window_workspace_bytes(1, 4, 2, 1, 100, 128, 10, 2) == 0
    assert L.ifa_window_workspace_bytes(1, 4, 3, 1, 100, 128, 10, 2) == -1 and L.ifa_window_workspace_bytes(1, 4, 2, 1, 100, 128, 0, 2) == -1


def test_prefix(L):
    for name in ("q", "kp", "vp", "k", "v", "sq", "skp", "sk", "o"):
        assert prefix(L, **{name: NULL}) == -1, name
    assert prefix(L, sv=P) == -1 and prefix(L, svp=P) == -1                # one of the two scales of V
    for bad in (dict(Np=0), dict(Np=-1), dict(H=3), dict(Nq=0), dict(Nk=0), dict(B=0)):
        assert prefix(L, **bad) == -2, bad
    assert prefix(L, dt=7) == -3
    for bad in (dict(d=256), dict(Np=0x7ff00000 // 256 + 1), dict(kp=ODD), dict(vp=ODD), dict(skp=ctypes.c_void_p(0x1001)), dict(Nq=1 << 25, Nk=1)):
        assert prefix(L, **bad) == -4, bad
    need = L.ifa_prefix_workspace_bytes(64, 32, 8, 1, 8192, 512, 128)
    assert need > 0
    big = dict(B=64, H=32, Hkv=8, Np=8192, Nk=512)
    assert prefix(L, **big, ws=NULL) == -1 and prefix(L, **big, n=need - 1) == -6 and prefix(L, **big, ws=ODD) == -4
    assert L.ifa_prefix_workspace_bytes(1, 4, 2, 1, 0, 100, 128) == -1


def weights(L, q=P, k=P, sq=P, sk=P, lens=NULL, w=NULL, B=1, H=4, Hkv=2, Nq=1, Nk=100, d=128, o=P, ws=WS, n=1 << 40):
    return L.key_weights(q, k, sq, sk, lens, w, B, H, Hkv, Nq, Nk, d, o, ws, n, None)


def test_key_weights(L):
    for name in ("q", "k", "sq", "sk", "o", "ws"):
        assert weights(L, **{name: NULL}) == -1, name
    for bad in (dict(B=0), dict(H=3), dict(Nq=0), dict(Nk=-1), dict(d=0)):
        assert weights(L, **bad) == -2, bad
    for bad in (dict(d=32), dict(q=ODD), dict(k=ODD), dict(ws=ODD), dict(w=ctypes.c_void_p(0x1002)), dict(o=ctypes.c_void_p(0x1002)), dict(Nk=0x7ff00000 // 256 + 1),
                dict(Nq=1 << 25, Nk=1), dict(B=1 << 10, H=2, Nk=1 << 20, d=64)):
        assert weights(L, **bad) == -4, bad
    assert weights(L, w=ctypes.c_void_p(0x1004)) == -4                     # W and W_out overlap, shifted
    need = L.ifa_key_weights_workspace_bytes(1, 4, 2, 1, 100, 128)
    assert need > 0 and weights(L, n=need - 1) == -6 and L.ifa_key_weights_workspace_bytes(1, 4, 2, 1, 100, 96) == -1


def evict(L, at=None, vb=2, lens=NULL, B=1, Hkv=2, Nk=100, d=128, keep=50, recent=5, sinks=4):
    """`at`: addresses of K, s_K, V, W and the six outputs."""
    a = [ctypes.c_void_p(x) for x in at or [(1 + i) << 20 for i in range(10)]]
    return L.evict_keys(a[0], a[1], a[2], vb, a[3], lens, B, Hkv, Nk, d, keep, recent, sinks, *a[4:], None)


def test_evict_keys(L):
    apart = [(1 + i) << 20 for i in range(10)]
    for i in range(10):
        assert evict(L, apart[:i] + [0] + apart[i + 1:]) == -1, i
    for bad in (dict(B=0), dict(Hkv=0), dict(Nk=0), dict(d=0), dict(keep=0), dict(keep=101), dict(recent=-1), dict(sinks=-1), dict(recent=30, sinks=21)):
        assert evict(L, **bad) == -2, bad
    assert evict(L, vb=4) == -3
    for bad in (dict(d=72), dict(d=1040), dict(B=1 << 22, Hkv=2, Nk=60, keep=50), dict(lens=ctypes.c_void_p(0x1002))):
        assert evict(L, **bad) == -4, bad
    for i in (0, 2, 4, 6):                               # K, V and their outputs: 16 bytes
        assert evict(L, apart[:i] + [apart[i] + 8] + apart[i + 1:]) == -4, i
    for i in range(4, 10):                               # an output on an input, on another output, or over the end of one
        for j in (0, 1, 2, 3, 4 + (i - 3) % 6):
            assert evict(L, apart[:i] + [apart[j]] + apart[i + 1:]) == -4, (i, j)
    assert evict(L, apart[:4] + [apart[0] + 2 * 100 * 128 - 16] + apart[5:]) == -4


def test_the_binding_names_the_operand(monkeypatch):
    q, k = torch.zeros(1, 4, 1, 64, dtype=torch.int8), torch.zeros(1, 2, 9, 64, dtype=torch.int8)
    v, sq, sk = torch.zeros(1, 2, 9, 64).half(), torch.ones(1, 4, 1), torch.ones(1, 2, 9)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    with pytest.raises(ifa.IntfaError, match="Q_i8: expected a contiguous tensor in GPU memory"):
        ifa.int_flash_attn_fwd_window(q, k, v, sq, sk, 4)
    with pytest.raises(ifa.IntfaError, match="do not agree"):
        ifa.int_flash_attn_fwd_window(q, torch.zeros(1, 3, 9, 64, dtype=torch.int8), v, sq, sk, 4)
    with pytest.raises(ifa.IntfaError, match="do not agree"):
        ifa.int_flash_attn_fwd_window(q, k[:, :, :0], v, sq, sk, 4)
    with pytest.raises(ifa.IntfaError, match="4-dimensional"):
        ifa.int_flash_attn_fwd_prefix(q, k[0], v[0], k[0], v, sq, sk[0], sk)
