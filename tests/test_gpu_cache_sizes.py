"""Evictions from caches of many layers, sequences and K/V heads."""
import pytest
import torch

from paper_2609_34977_gb300 import _native as N

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("L,B,G,n,budget", [(32, 64, 32, 3, 2), (32, 64, 32, 140, 70), (4, 300, 60, 3, 2)])
def test_eviction_from_more_than_65535_units(L, B, G, n, budget):
    # moves in the selecting kernel and in one of their own. Weights rise with the slot in even units, which keep their last
    # rows, and fall in odd ones, where nothing moves
    d, slots = 64, n + 1
    g = torch.Generator(device="cuda").manual_seed(n)
    kv = torch.randint(-30000, 30000, (L, B, slots, 2, G, d), dtype=torch.int16, device="cuda", generator=g)
    unit = torch.arange(L * B * G, device="cuda").view(L, B, G, 1)
    slot = torch.arange(slots, device="cuda")
    acc = torch.where(unit % 2 == 0, slot, -slot).float()
    src = torch.where(unit % 2 == 0, torch.where(slot < n - budget, slot + budget, slot), slot)[..., :budget]
    at = src.permute(0, 1, 3, 2)[:, :, :, None, :, None].expand(L, B, budget, 2, G, d)
    want = kv.clone()
    want[:, :, :budget] = torch.gather(kv, 2, at)
    want_acc = torch.cat([torch.gather(acc, 3, src), torch.zeros_like(acc[..., budget:n]), acc[..., n:]], 3)
    got_src = torch.full((L, B, G, budget), -3, dtype=torch.int32, device="cuda")
    ws = torch.zeros(N.spd_cache_evict_workspace_size(L, B, G, budget), dtype=torch.uint8, device="cuda")
    N.spd_cache_evict(kv.view(torch.bfloat16), [n] * B, slots, G, d, budget, 0, 0, None, acc, None, acc, None, got_src, ws)
    assert torch.equal(got_src, src.int())
    assert torch.equal(kv, want) and torch.equal(acc, want_acc)
