"""The largest grids of the calls on a quantized cache: a launch has less than 2^32 threads, and a call that would need more is refused on the host."""
import ctypes

import pytest
import torch

import paper_2409_16997_amd as ifa

AT = [ctypes.c_void_p((1 + i) << 40) for i in range(10)]         # K, s_K, V, W and the six outputs, far apart


def evict(B, Hkv, Nk=2, d=16, keep=1):
    return ifa.lib().evict_keys(*AT[:3], 1, AT[3], None, B, Hkv, Nk, d, keep, 0, 0, *AT[4:], None)


def test_an_eviction_of_more_heads_than_a_launch_has_workgroups_is_refused():
    """A workgroup of 1024 threads to a key head: 2^22 of them are one too many."""
    assert evict(1 << 11, 1 << 11) == -4
    assert evict((1 << 22) + 1, 1) == -4


@pytest.mark.gpu
def test_an_eviction_of_as_many_heads_as_a_launch_has_workgroups():
    heads = (1 << 22) - 1
    g = torch.Generator(device="cuda").manual_seed(4)
    k8 = torch.randint(-127, 128, (1, heads, 2, 16), dtype=torch.int8, device="cuda", generator=g)
    sk = torch.rand((1, heads, 2), device="cuda", generator=g)
    W = torch.rand((1, heads, 2), device="cuda", generator=g)
    k, s, v, w, index, left = ifa.evict_keys(k8, sk, k8, W, 1)
    best = W.argmax(2, keepdim=True)
    assert torch.equal(index.long(), best) and torch.equal(w, W.gather(2, best)) and torch.equal(s, sk.gather(2, best)) and left.tolist() == [1]
    row = k8.gather(2, best.unsqueeze(-1).expand(1, heads, 1, 16))
    assert torch.equal(k, row) and torch.equal(v, row)
