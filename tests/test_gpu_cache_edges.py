"""Attention over a cache where its slots end: full caches at the end of their
buffer, weights summed in place by every form of the weights' pass, slots that a
window hides. Against the float64 oracle with the tolerances of the cache's other
tests, or equal to the bit."""
import math

import pytest
import torch

import paper_2609_23169_amd as ut
from test_gpu_cache import check_attn, dev, rnd

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("cap", [1, 10, 33, 47, 300, 5003])
@pytest.mark.parametrize("Hq,Hk,D", [(4, 4, 64), (4, 1, 128), (64, 2, 40)])
def test_full_caches_of_any_length(cap, Hq, Hk, D):
    """The last step of 32 slots is cut at any of them, and the last sample's at the
    end of the buffer; what follows a single cache in memory changes nothing."""
    B, T = 2, 1
    q, k, v = rnd(1, B, T, Hq, D), rnd(2, B, cap, Hk, D), rnd(3, B, cap, Hk, D)
    w = torch.rand((B, Hk, cap), device=DEV)
    o, lse, got = ut.cache_attn(q, k, v, dev([cap - 1] * B), D ** -0.5, weights=w)
    check_attn(q, k, v, [cap - 1] * B, D ** -0.5, o, lse, None, None, 0, w, got)
    more = [torch.full((1, cap + 64, Hk, D), math.nan, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    for x, y in zip(more, (k, v)):
        x[:, :cap] = y[1:]
    alone = ut.cache_attn(q[1:], *(x[:, :cap] for x in more), dev([cap - 1]), D ** -0.5, weights=w[1:])
    want = ut.cache_attn(q[1:], k[1:], v[1:], dev([cap - 1]), D ** -0.5, weights=w[1:])
    for x, y in zip(alone, want):
        assert torch.equal(x, y)


def test_eviction_into_neighbouring_views_of_one_buffer():
    B, cap, Hk, D, keep, lens = 2, 300, 2, 64, 100, [300, 70]
    k, v, w = rnd(4, B, cap, Hk, D), rnd(5, B, cap, Hk, D), torch.rand((B, Hk, cap), device=DEV)
    want = ut.cache_evict(k, v, w, dev(lens), keep, 2, 9)
    for first, second, count in ((0, 1, 2), (1, 0, 2), (2, 1, 3)):
        kv = torch.empty((B, keep, count, Hk, D), dtype=torch.bfloat16, device=DEV)
        wo, lo, idx = (torch.empty_like(x) for x in want[2:])
        assert ut.ut_cache_evict(k, v, w, dev(lens), kv[:, :, first], kv[:, :, second], wo, lo, idx, keep, 2, 9) == ut.UT_OK
        for x, y in zip((kv[:, :, first], kv[:, :, second], wo, lo, idx), want):
            assert torch.equal(x, y)
