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


@pytest.mark.parametrize("T,Hq,Hk", [(1, 8, 2), (20, 4, 2), (40, 4, 2), (140, 2, 1)])
@pytest.mark.parametrize("cap,left,sinks", [(3000, None, 0), (9000, 1000, 3)])
def test_weights_in_place_are_those_out_of_place(T, Hq, Hk, cap, left, sinks):
    """From the scores of few rows and by the pass over the keys, by the capacity and
    (the window) shared out by what is seen, where unseen slots depend on whether there is
    something to copy."""
    B, D = 2, 64
    q, k, v = rnd(6, B, T, Hq, D), rnd(7, B, cap, Hk, D), rnd(8, B, cap, Hk, D)
    lens, w = dev([cap - T, cap // 3]), torch.rand((B, Hk, cap), device=DEV)
    at = dict(window_left=left, n_sink=sinks)
    o, lse, want = ut.cache_attn(q, k, v, lens, 0.125, weights=w, **at)
    check_attn(q, k, v, lens.tolist(), 0.125, o, lse, None, left, sinks, w, want)
    mine = w.clone()
    ut.cache_attn(q, k, v, lens, 0.125, weights=mine, weights_out=mine, **at)
    assert torch.equal(mine, want)
    alone = ut.cache_weights(q, k, lse, lens, 0.125, weights=w, **at)
    check_attn(q, k, v, lens.tolist(), 0.125, o, lse, None, left, sinks, w, alone)
    mine = w.clone()
    ut.cache_weights(q, k, lse, lens, 0.125, weights=mine, weights_out=mine, **at)
    assert torch.equal(mine, alone)
    # from nothing, into what may hold anything
    zero, junk = torch.zeros_like(w), torch.full_like(w, math.nan)
    assert torch.equal(ut.cache_weights(q, k, lse, lens, 0.125, weights_out=junk, **at),
                       ut.cache_weights(q, k, lse, lens, 0.125, weights=zero, **at))


@pytest.mark.parametrize("T", [40, 250])
def test_shared_out_steps_beyond_one_turn(T):
    """2,560 steps of four tiles and more on 256 workgroups: more than the eight that a wave
    keeps sums of at once, within an item and across items; 250 rows in two loads."""
    B, H, cap, D, left = 16, 16, 6100, 64, 2200
    q, k, v = rnd(9, B, T, H, D), rnd(10, B, cap, H, D), rnd(11, B, cap, H, D)
    lens = [cap - T - 37 * b for b in range(B)]
    lens[3], lens[9] = 0, 2000
    w = torch.rand((B, H, cap), device=DEV)
    o, lse, got = ut.cache_attn(q, k, v, dev(lens), D ** -0.5, window_left=left, n_sink=70, weights=w)
    alone = ut.cache_weights(q, k, lse, dev(lens), D ** -0.5, window_left=left, n_sink=70, weights=w)
    for b, h in ((0, 0), (0, 15), (3, 7), (7, 2), (9, 11), (15, 15)):
        s, c = slice(b, b + 1), slice(h, h + 1)
        for x in (got, alone):
            check_attn(q[s, :, c], k[s, :, c], v[s, :, c], [lens[b]], D ** -0.5, o[s, :, c], lse[s, c], None, left, 70, w[s, c], x[s, c])


@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("T,Hq,Hk,D", [(1, 8, 2, 64), (5, 4, 1, 128), (40, 4, 2, 64), (140, 1, 1, 128)])
def test_slots_in_front_of_every_window_may_hold_anything(bad, T, Hq, Hk, D):
    B, cap, lens, left, sinks = 2, 4000, [3800, 700], 300, 3
    q, k, v, w = rnd(12, B, T, Hq, D), rnd(13, B, cap, Hk, D), rnd(14, B, cap, Hk, D), torch.rand((B, Hk, cap), device=DEV)
    at = dict(window_left=left, n_sink=sinks, weights=w)
    want = ut.cache_attn(q, k, v, dev(lens), 0.1, **at)
    alone = ut.cache_weights(q, k, want[1], dev(lens), 0.1, **at)
    for b, n in enumerate(lens):
        for x in (k, v):
            x[b, sinks:n - left], x[b, n + T:] = bad, bad
    for x, y in zip(ut.cache_attn(q, k, v, dev(lens), 0.1, **at), want):
        assert torch.equal(x, y)
    assert torch.equal(ut.cache_weights(q, k, want[1], dev(lens), 0.1, **at), alone)


@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("T", [6, 40])
def test_a_hidden_tokens_key_may_hold_anything(bad, T):
    """The last drafted token, seen by itself alone: its key reaches no other token, and
    with its value left finite neither does anything else of it."""
    B, cap, lens = 1, 500, [400]
    q, k, v = rnd(15, B, T, 4, 64), rnd(16, B, cap, 2, 64), rnd(17, B, cap, 2, 64)
    tree = dev([[(1 << t + 1) - 1 for t in range(T - 1)] + [1 << T - 1]], torch.int64)
    want = ut.cache_attn(q, k, v, dev(lens), 0.1, tree=tree)
    k[0, lens[0] + T - 1] = bad
    got = ut.cache_attn(q, k, v, dev(lens), 0.1, tree=tree)
    assert torch.equal(got[0][:, :T - 1], want[0][:, :T - 1]) and torch.equal(got[1][:, :, :T - 1], want[1][:, :, :T - 1])
