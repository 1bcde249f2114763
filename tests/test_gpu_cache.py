"""Attention over a cache, the weights that its slots receive, and eviction, on the
GPU against the float64 oracle; and the three together as a generating model uses
them.

Tolerances of the attention: those of the window attention's tests. Weights are
sums in fp32 of P = exp(S scale - LSE) with both in fp32: with x as there (scores and
exponential) and the LSE's own tolerance, P is off by 2 x + 2^-22 max(1, |LSE|) of
itself, and a sum of n terms by n 2^-24 more. Eviction copies: equal to the bit."""
import math

import numpy as np
import pytest
import torch

import oracle
import paper_2609_23169_amd as ut
from test_gpu_swattn import E24, check_head, f64

pytestmark = pytest.mark.gpu
DEV = "cuda"


def dev(x, dtype=torch.int32):
    return torch.tensor(x, dtype=dtype, device=DEV)


def rnd(seed, *shape):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(shape, generator=g).to(torch.bfloat16).to(DEV)


def words(seed, B, T, tree=True):
    """Random trees (an ancestor's bits and the token's own), or any bits at all."""
    rng = np.random.default_rng(seed)
    out = np.zeros((B, T), np.uint64)
    for b in range(B):
        for t in range(T):
            if not tree:
                out[b, t] = rng.integers(0, 1 << 63, dtype=np.uint64) * np.uint64(rng.integers(0, 2))
            else:
                parent = int(rng.integers(-1, t)) if t else -1
                out[b, t] = (out[b, parent] if parent >= 0 else np.uint64(0)) | np.uint64(1) << np.uint64(t)
    return out


def check_attn(q, k, v, lens, scale, o, lse, tree=None, left=None, sinks=0, w_in=None, w=None, tokens=None, label=""):
    B, T, Hq, D = q.shape
    cap, Hk = k.shape[1], k.shape[2]
    G = Hq // Hk
    Q, K, V = f64(q), f64(k), f64(v)
    O, L, W = oracle.cache_attn(Q, K, V, lens, scale, tree, left, sinks, tokens)
    tol = np.zeros(W.shape)
    for b in range(B):
        see = oracle.cache_see(T, cap, int(lens[b]), None if tree is None else tree[b], left, sinks)
        for h in range(Hq):
            P, x, _, _, _ = check_head(Q[b, :, h], K[b, :, h // G], V[b, :, h // G], see, scale, O[b, :, h], L[b, h],
                                       f64(o)[b, :, h], f64(lse)[b, h], label, D)
            far = np.where(np.isfinite(L[b, h]), np.abs(L[b, h]), 0)[:, None]
            tol[b, h // G] += (P * (2 * x + 2.0 ** -22 * np.maximum(1, far))).sum(0)
    if w is not None:
        base = 0.0 if w_in is None else f64(w_in)
        tol += (T * G + 2) * E24 * (W + np.abs(base))
        err = np.abs(f64(w) - (base + W))
        assert np.all(err <= tol), (label, "weights", float((err / (tol + 1e-30)).max()))
        if tokens is None:
            seen = (f64(w) - base).sum(2)
            assert np.all(seen <= T * G + 1e-3)


CASES = [  # B, T, cap, lens, Hq, Hk, D, left, sinks
    (1, 1, 1, [0], 1, 1, 64, None, 0), (1, 1, 300, [200], 8, 2, 64, None, 0), (3, 1, 700, [0, 699, 64], 4, 1, 128, None, 0),
    (2, 1, 5000, [4999, 3000], 8, 2, 128, None, 0), (2, 1, 3000, [2999, 100], 8, 2, 64, 500, 4),
    (1, 1, 2000, [1500], 40, 1, 128, 63, 1), (2, 5, 400, [395, 0], 4, 2, 40, None, 0), (1, 64, 500, [300], 4, 4, 128, 70, 2),
    (2, 200, 1500, [1300, 33], 2, 1, 64, None, 0), (1, 130, 130, [0], 3, 3, 72, 20, 5), (2, 33, 4300, [4200, 64], 6, 2, 96, 1000, 100),
    (1, 3, 64, [61], 5, 5, 8, 0, 0),
]


@pytest.mark.parametrize("B,T,cap,lens,Hq,Hk,D,left,sinks", CASES)
def test_chains_match_oracle(B, T, cap, lens, Hq, Hk, D, left, sinks):
    q, k, v = rnd(1, B, T, Hq, D), rnd(2, B, cap, Hk, D), rnd(3, B, cap, Hk, D)
    w = torch.rand((B, Hk, cap), device=DEV)
    o, lse, got = ut.cache_attn(q, k, v, dev(lens), D ** -0.5, window_left=left, n_sink=sinks, weights=w)
    check_attn(q, k, v, lens, D ** -0.5, o, lse, None, left, sinks, w, got)


@pytest.mark.parametrize("kind", ["tree", "any"])
@pytest.mark.parametrize("B,T,cap,lens,Hq,Hk,D,left,sinks", [
    (1, 1, 10, [4], 2, 1, 64, None, 0), (2, 7, 300, [293, 0], 4, 2, 128, None, 0), (1, 64, 64, [0], 2, 2, 64, None, 0),
    (2, 64, 2000, [1936, 700], 4, 1, 128, 300, 3), (3, 33, 500, [60, 31, 467], 6, 2, 72, 32, 0), (1, 48, 9000, [8900], 8, 2, 128, None, 0),
    (2, 20, 300, [2, 100], 2, 2, 64, 40, 10),
])
def test_trees_match_oracle(B, T, cap, lens, Hq, Hk, D, left, sinks, kind):
    q, k, v = rnd(4, B, T, Hq, D), rnd(5, B, cap, Hk, D), rnd(6, B, cap, Hk, D)
    tree = words(7, B, T, kind == "tree")
    t = torch.from_numpy(tree.view(np.int64)).to(DEV)
    w = torch.rand((B, Hk, cap), device=DEV)
    o, lse, got = ut.cache_attn(q, k, v, dev(lens), D ** -0.5, tree=t, window_left=left, n_sink=sinks, weights=w)
    check_attn(q, k, v, lens, D ** -0.5, o, lse, tree, left, sinks, w, got, label=kind)
    picked = words(8, B, 1, False)[:, 0] | np.uint64(1)
    got = ut.cache_weights(q, k, lse, dev(lens), D ** -0.5, tree=t, tokens=torch.from_numpy(picked.view(np.int64)).to(DEV),
                           window_left=left, n_sink=sinks)
    check_attn(q, k, v, lens, D ** -0.5, o, lse, tree, left, sinks, None, got, picked, label=kind)


def test_a_chain_as_a_tree_is_the_chain():
    B, T, cap, lens = 2, 19, 400, [381, 50]
    q, k, v = rnd(9, B, T, 4, 64), rnd(10, B, cap, 2, 64), rnd(11, B, cap, 2, 64)
    tree = dev([[(1 << t + 1) - 1 for t in range(T)]] * B, torch.int64)
    for left in (None, 18, 100):
        a = ut.cache_attn(q, k, v, dev(lens), 0.125, window_left=left, n_sink=3)
        b = ut.cache_attn(q, k, v, dev(lens), 0.125, tree=tree, window_left=left, n_sink=3)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_a_chain_equals_window_attention():
    B, T, n = 2, 100, 300
    q, k, v = rnd(12, B, T, 4, 128), rnd(13, B, n + T, 2, 128), rnd(14, B, n + T, 2, 128)
    a = ut.cache_attn(q, k, v, dev([n, n]), 0.1, window_left=80, n_sink=4)
    b = ut.swattn_fwd(q, k, v, (80, 0), 0.1, 4)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("T", [1, 40])
def test_slots_not_in_use_may_hold_anything(bad, T):
    B, cap, lens = 2, 500, [333, 60]
    q, k, v, w = rnd(15, B, T, 4, 64), rnd(16, B, cap, 2, 64), rnd(17, B, cap, 2, 64), torch.rand((B, 2, cap), device=DEV)
    a = ut.cache_attn(q, k, v, dev(lens), 0.125, weights=w)
    for b, n in enumerate(lens):
        k[b, n + T:], v[b, n + T:] = bad, bad
    b = ut.cache_attn(q, k, v, dev(lens), 0.125, weights=w)
    for x, y in zip(a, b):
        assert torch.equal(x, y)
    for i, n in enumerate(lens):
        assert torch.equal(a[2][i, :, n + T:], w[i, :, n + T:])


def test_lengths_out_of_range_are_clamped():
    B, T, cap = 3, 2, 100
    q, k, v, w = rnd(18, B, T, 2, 64), rnd(19, B, cap, 1, 64), rnd(20, B, cap, 1, 64), torch.rand((B, 1, cap), device=DEV)
    a = ut.cache_attn(q, k, v, dev([-5, 1000, 98]), 0.125, weights=w)
    b = ut.cache_attn(q, k, v, dev([0, 98, 98]), 0.125, weights=w)
    for x, y in zip(a, b):
        assert torch.equal(x, y)


def test_weights_in_place_and_from_nothing():
    q, k, v = rnd(21, 2, 1, 8, 64), rnd(22, 2, 3000, 2, 64), rnd(23, 2, 3000, 2, 64)
    lens, w = dev([2999, 1000]), torch.rand((2, 2, 3000), device=DEV)
    o, lse, want = ut.cache_attn(q, k, v, lens, 0.125, weights=w)
    alone = torch.full_like(w, math.nan)
    o2, lse2, got = ut.cache_attn(q, k, v, lens, 0.125, weights_out=alone)
    assert torch.equal(o, o2) and torch.equal(lse, lse2) and got is alone
    assert torch.allclose(w + alone, want, rtol=2.0 ** -22)
    # from the scores and formed again: each off by 2 x + 2^-22 |LSE| of itself, A = sum|q k| scale below 12
    assert torch.allclose(ut.cache_weights(q, k, lse, lens, 0.125), alone, rtol=2 * (2 * (2 * 72 * 12 * E24 + 2.0 ** -18) + 2.0 ** -19),
                          atol=0)
    mine = w.clone()
    ut.cache_attn(q, k, v, lens, 0.125, weights=mine, weights_out=mine)
    assert torch.equal(mine, want)
    assert len(ut.cache_attn(q, k, v, lens, 0.125)) == 2
    none = ut.cache_weights(q, k, lse, lens, 0.125, weights=w, tokens=dev([0, 0], torch.int64))
    assert torch.equal(none, w)


def test_slots_past_32_bit_offsets():
    cap, stride, D, n = 700, (1 << 22) - 8, 64, 650
    q, k, v = rnd(24, 1, 1, 4, D), rnd(25, 1, cap, 1, D), rnd(26, 1, cap, 1, D)
    buf = torch.empty((cap - 1) * stride + 2 * D, dtype=torch.bfloat16, device=DEV)
    kf = torch.as_strided(buf, (1, cap, 1, D), (cap * stride, stride, D, 1))
    vf = torch.as_strided(buf, (1, cap, 1, D), (cap * stride, stride, D, 1), D)
    kf.copy_(k), vf.copy_(v)
    w = torch.rand((1, 1, cap), device=DEV)
    a, b = (ut.cache_attn(q, *x, dev([n]), 0.125, weights=w) for x in ((k, v), (kf, vf)))
    for x, y in zip(a, b):
        assert torch.equal(x, y)
    a, b = (ut.cache_evict(*x, w, dev([n]), 300, 4, 10) for x in ((k, v), (kf, vf)))
    for x, y in zip(a, b):
        assert torch.equal(x, y)


# ---- eviction --------------------------------------------------------------

def check_evict(k, v, w, lens, keep, sinks, recent, got, capacity=None):
    ko, vo, wo, lo, idx = got
    B, cap, Hk, D = k.shape
    assert lo.tolist() == [min(n, keep) for n in lens]
    for b in range(B):
        m = min(lens[b], keep)
        for h in range(Hk):
            want = oracle.cache_evict(w[b, h].cpu().numpy(), lens[b], keep, sinks, recent)
            assert idx[b, h, :m].tolist() == want.tolist(), (b, h)
            at = torch.from_numpy(want).to(DEV)
            assert torch.equal(ko[b, :m, h], k[b, at, h]) and torch.equal(vo[b, :m, h], v[b, at, h])
            assert torch.equal(wo[b, h, :m].view(torch.int32), w[b, h, at].view(torch.int32))
        assert (idx[b, :, m:] == -1).all() and (wo[b, :, m:] == 0).all()
        assert (ko[b, m:] == 0).all() and (vo[b, m:] == 0).all()


def weights(seed, kind, *shape):
    g = torch.Generator().manual_seed(seed)
    w = torch.randn(shape, generator=g)
    if kind == "ties":
        w = (w * 2).round() / 4
    elif kind == "equal":
        w = torch.zeros(shape)
        w.view(-1)[::2] = -0.0
    elif kind == "special":
        w.view(-1)[::7], w.view(-1)[1::11], w.view(-1)[2::13], w.view(-1)[3::17] = math.nan, math.inf, -math.inf, -0.0
    elif kind == "nan":
        w = torch.full(shape, math.nan)
    elif kind == "tiny":
        w = w * 1e-42       # denormal
    elif kind == "sums":
        w = (w * 2).exp() * (torch.rand(shape, generator=g) > 0.1)
    return w.to(DEV)


@pytest.mark.parametrize("kind", ["plain", "ties", "equal", "special", "nan", "tiny", "sums"])
@pytest.mark.parametrize("cap,lens,keep,sinks,recent", [
    (300, [300, 120, 0], 128, 4, 32), (2000, [2000, 1999, 700], 699, 0, 0), (5000, [4999, 64, 4100], 1000, 4, 900),
])
def test_eviction_by_kinds_of_weights(kind, cap, lens, keep, sinks, recent):
    k, v = rnd(27, 3, cap, 2, 64), rnd(28, 3, cap, 2, 64)
    w = weights(29, kind, 3, 2, cap)
    check_evict(k, v, w, lens, keep, sinks, recent, ut.cache_evict(k, v, w, dev(lens), keep, sinks, recent))


@pytest.mark.parametrize("cap,lens,keep,sinks,recent,Hk,D", [
    (1, [1], 1, 0, 0, 1, 8), (2, [2, 1], 1, 1, 0, 1, 64), (2, [2, 2], 1, 0, 1, 3, 128), (65, [65], 64, 10, 54, 1, 40),
    (65, [65], 64, 10, 53, 2, 40), (4096, [4096], 4095, 0, 0, 1, 64), (4200, [4200], 1, 0, 0, 1, 64), (17000, [16999, 5], 4096, 4, 1000, 2, 128),
    (33000, [33000], 300, 1, 0, 1, 64), (70001, [70001, 66000], 20000, 64, 256, 1, 16), (68000, [68000, 33000, 40], 20000, 4, 256, 1, 16), (500, [400, 500], 500, 4, 4, 2, 96),
    (20000, [20000], 12345, 7, 333, 5, 24),
])
def test_eviction_by_sizes(cap, lens, keep, sinks, recent, Hk, D):
    B = len(lens)
    k, v = rnd(30, B, cap, Hk, D), rnd(31, B, cap, Hk, D)
    for kind in ("sums", "ties"):
        w = weights(32, kind, B, Hk, cap)
        check_evict(k, v, w, lens, keep, sinks, recent, ut.cache_evict(k, v, w, dev(lens), keep, sinks, recent))


def test_eviction_into_a_larger_cache_and_views():
    """Rows behind n_keep stay, or become 0; interleaved caches in and out."""
    B, cap, Hk, D, keep, lens = 2, 400, 2, 64, 100, [400, 60]
    kv = rnd(33, B, cap, 2, Hk, D)
    w = weights(34, "sums", B, Hk, cap)
    out = torch.full((B, 150, 3, Hk, D), 5.0, dtype=torch.bfloat16, device=DEV)
    wo, lo = torch.full((B, Hk, 150), 5.0, device=DEV), torch.full((B,), 5, dtype=torch.int32, device=DEV)
    idx = torch.empty((B, Hk, keep), dtype=torch.int32, device=DEV)
    k, v = kv[:, :, 0], kv[:, :, 1]
    for zero in (False, True):
        assert ut.ut_cache_evict(k, v, w, dev(lens), out[:, :, 0], out[:, :, 2], wo, lo, idx, keep, 4, 10, zero) == ut.UT_OK
        check_evict(k, v, w, lens, keep, 4, 10, (out[:, :keep, 0], out[:, :keep, 2], wo[:, :, :keep], lo, idx))
        assert (out[:, :, 1] == 5).all() and (wo[:, :, keep:] == 0).all()
        assert (out[:, keep:, 0] == (0 if zero else 5)).all() and (out[:, keep:, 2] == (0 if zero else 5)).all()
    got = ut.cache_evict(k, v, w, dev(lens), keep, 4, 10, capacity=170)
    assert got[0].shape == (B, 170, Hk, D) and (got[0][:, keep:] == 0).all() and got[2].shape == (B, Hk, 170)
    assert torch.equal(got[0][:, :keep], out[:, :keep, 0])


def test_eviction_of_lengths_out_of_range():
    k, v, w = rnd(35, 2, 200, 1, 64), rnd(36, 2, 200, 1, 64), weights(37, "sums", 2, 1, 200)
    got = ut.cache_evict(k, v, w, dev([-3, 5000]), 50, 1, 2)
    check_evict(k, v, w, [0, 200], 50, 1, 2, got)


# ---- together --------------------------------------------------------------

def test_generation_with_eviction_and_a_tree():
    """A prompt in two chunks, tokens one by one with their weights, eviction, more
    tokens, then a drafted tree of which a path is accepted: every step against
    the oracle on what the step before left."""
    B, Hq, Hk, D, cap = 2, 4, 2, 64, 260
    scale, rng = D ** -0.5, np.random.default_rng(40)
    k, v = (torch.full((B, cap, Hk, D), math.nan, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    w, lens, seed = torch.zeros((B, Hk, cap), device=DEV), [0, 0], [100]

    def put(T):
        seed[0] += 3
        kn, vn = rnd(seed[0], B, T, Hk, D), rnd(seed[0] + 1, B, T, Hk, D)
        for b in range(B):
            k[b, lens[b]:lens[b] + T], v[b, lens[b]:lens[b] + T] = kn[b], vn[b]
        return rnd(seed[0] + 2, B, T, Hq, D)

    def step(T, tree=None, count=True):
        nonlocal w
        q = put(T)
        t = None if tree is None else torch.from_numpy(tree.view(np.int64)).to(DEV)
        got = ut.cache_attn(q, k, v, dev(lens), scale, tree=t, weights=w if count else None)
        check_attn(q, torch.nan_to_num(k), torch.nan_to_num(v), lens, scale, got[0], got[1], tree, None, 0, w,
                   got[2] if count else None)
        if count:
            w = got[2]
        return q, got[1], t

    for T in (100, 53):
        step(T)
        lens = [n + T for n in lens]
    for _ in range(3):
        step(1)
        lens = [n + 1 for n in lens]
    ko, vo, wo, lo, idx = ut.cache_evict(k, v, w, dev(lens), 80, 4, 16, capacity=cap)
    check_evict(k, v, w, lens, 80, 4, 16, (ko[:, :80], vo[:, :80], wo[:, :, :80], lo, idx))
    k, v, w, lens = ko, vo, wo, lo.tolist()
    assert lens == [80, 80]
    step(1)
    lens = [n + 1 for n in lens]
    T = 12
    tree = words(41, B, T)
    q, lse, t = step(T, tree, count=False)
    accepted = np.array([tree[b, int(rng.integers(0, T))] for b in range(B)])      # a token and its ancestors
    got = ut.cache_weights(q, k, lse, dev(lens), scale, weights=w, tree=t,
                           tokens=torch.from_numpy(accepted.view(np.int64)).to(DEV))
    W = oracle.cache_attn(f64(q), f64(torch.nan_to_num(k)), f64(torch.nan_to_num(v)), lens, scale, tree, tokens=accepted)[2]
    assert np.abs(f64(got) - f64(w) - W).max() <= 1e-4 * W.max()
    for b in range(B):
        path = [u for u in range(T) if int(accepted[b]) >> u & 1]
        rows = dev([lens[b] + u for u in path], torch.int64)
        k[b, lens[b]:lens[b] + len(path)], v[b, lens[b]:lens[b] + len(path)] = k[b, rows], v[b, rows]
        lens[b] += len(path)
    w = got
    step(1)


def test_captured_and_replayed():
    """A decoding step and an eviction in a graph: lengths and weights are read at
    every replay."""
    B, Hq, Hk, D, cap = 2, 8, 2, 128, 5000
    q, k, v = rnd(50, B, 1, Hq, D), rnd(51, B, cap, Hk, D), rnd(52, B, cap, Hk, D)
    lens, w = dev([4000, 100]), torch.rand((B, Hk, cap), device=DEV)
    w2, l2 = w.clone(), lens.clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o, lse, _ = ut.cache_attn(q, k, v, l2, 0.1, weights=w2, weights_out=w2)
        kept = ut.cache_evict(k, v, w2, l2, 600, 4, 64)
    for n in ([4000, 100], [4999, 4998], [0, 700]):
        l2.copy_(dev(n))
        w2.copy_(w)
        graph.replay()
        a = ut.cache_attn(q, k, v, dev(n), 0.1, weights=w)
        b = ut.cache_evict(k, v, a[2], dev(n), 600, 4, 64)
        torch.cuda.synchronize()
        for x, y in zip((o, lse, w2) + kept, a + b):
            assert torch.equal(x, y)


def test_on_another_stream():
    q, k, v = rnd(53, 2, 1, 8, 128), rnd(54, 2, 6000, 2, 128), rnd(55, 2, 6000, 2, 128)
    lens, w = dev([5000, 5999]), torch.rand((2, 2, 6000), device=DEV)
    want = ut.cache_attn(q, k, v, lens, 0.1, weights=w)
    want += ut.cache_evict(k, v, want[2], lens, 1000, 4, 64)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = ut.cache_attn(q, k, v, lens, 0.1, weights=w, stream=s)
    got += ut.cache_evict(k, v, got[2], lens, 1000, 4, 64, stream=s)
    s.synchronize()
    for x, y in zip(got, want):
        assert torch.equal(x, y)
