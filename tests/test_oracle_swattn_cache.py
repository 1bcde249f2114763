"""The oracle of window attention, attention over a cache and eviction: against
definitions written out pair by pair, identities and central differences."""
import math

import numpy as np
import pytest

import oracle


def _rand(seed, *shape):
    return np.random.default_rng(seed).standard_normal(shape)


def test_window_by_hand():
    see = oracle.window_see(4, 4, 1, 0, 1)
    assert see.astype(int).tolist() == [[1, 0, 0, 0], [1, 1, 0, 0], [1, 1, 1, 0], [1, 0, 1, 1]]
    see = oracle.window_see(4, 4, 0, 1, 2)     # looks ahead: the two sinks are seen by all
    assert see.astype(int).tolist() == [[1, 1, 0, 0], [1, 1, 1, 0], [1, 1, 1, 1], [1, 1, 0, 1]]
    see = oracle.window_see(2, 5, 1, 0)        # two queries at the end of five keys
    assert see.astype(int).tolist() == [[0, 0, 1, 1, 0], [0, 0, 0, 1, 1]]
    assert not oracle.window_see(3, 1, 5, 0)[:2].any()          # queries in front of the keys
    assert oracle.window_see(7, 9, None, None).all()


@pytest.mark.parametrize("left,right,sinks", [(3, 0, 2), (2, 4, 0), (0, 0, 0), (None, 0, 0), (5, None, 1)])
def test_window_attention_pair_by_pair(left, right, sinks):
    B, Nq, Nk, Hq, Hk, D, scale = 2, 7, 11, 4, 2, 3, 0.7
    q, k, v = _rand(1, B, Nq, Hq, D), _rand(2, B, Nk, Hk, D), _rand(3, B, Nk, Hk, D)
    mask = np.random.default_rng(4).random((B, Nk)) < 0.7
    O, L = oracle.swattn_fwd(q, k, v, scale, left, right, sinks, mask)
    for b in range(B):
        for h in range(Hq):
            for i in range(Nq):
                p, w, o = i + Nk - Nq, 0.0, np.zeros(D)
                for j in range(Nk):
                    near = (left is None or p - j <= left) and (right is None or j - p <= right)
                    sink = j < sinks and (right != 0 or j <= p)
                    if mask[b, j] and (near or sink):
                        e = math.exp(scale * float(q[b, i, h] @ k[b, j, h // 2]))
                        w, o = w + e, o + e * v[b, j, h // 2]
                if w == 0:
                    assert L[b, h, i] == -np.inf and not O[b, i, h].any()
                else:
                    assert abs(L[b, h, i] - math.log(w)) < 1e-12 and np.allclose(O[b, i, h], o / w, atol=1e-12)


def test_window_attention_without_bounds_is_cross_attention():
    q, k, v, do = _rand(1, 2, 5, 4, 8), _rand(2, 2, 9, 2, 8), _rand(3, 2, 9, 2, 8), _rand(4, 2, 5, 4, 8)
    mask = np.random.default_rng(5).random((2, 9)) < 0.6
    for x, y in zip(oracle.swattn_fwd(q, k, v, 0.3, None, None, 0, mask) + oracle.swattn_bwd(q, k, v, do, 0.3, None, None, 0, mask),
                    oracle.xattn_fwd(q, k, v, 0.3, mask) + oracle.xattn_bwd(q, k, v, do, 0.3, mask)):
        assert np.allclose(x, y, atol=1e-13)


def test_window_gradients_by_differences():
    q, k, v, do = _rand(1, 1, 6, 2, 3), _rand(2, 1, 6, 1, 3), _rand(3, 1, 6, 1, 3), _rand(4, 1, 6, 2, 3)
    args = (0.5, 2, 0, 1)
    grads = oracle.swattn_bwd(q, k, v, do, *args)
    for n, x in enumerate((q, k, v)):
        for at in np.ndindex(x.shape):
            y = [[q, k, v][m].copy() for m in range(3)]
            y[n][at] += 1e-5
            up = (oracle.swattn_fwd(*y, *args)[0] * do).sum()
            y[n][at] -= 2e-5
            down = (oracle.swattn_fwd(*y, *args)[0] * do).sum()
            assert abs((up - down) / 2e-5 - grads[n][at]) < 1e-7


def test_cache_tokens_equal_the_last_rows_of_window_attention():
    B, T, cap, Hq, Hk, D = 2, 4, 20, 4, 2, 8
    q, k, v = _rand(1, B, T, Hq, D), _rand(2, B, cap, Hk, D), _rand(3, B, cap, Hk, D)
    for left, sinks in ((None, 0), (3, 2), (2, 0)):
        lens = [11, 0]
        O, L, W = oracle.cache_attn(q, k, v, lens, 0.4, None, left, sinks)
        for b, n in enumerate(lens):
            o, l = oracle.swattn_fwd(q[b:b + 1], k[b:b + 1, :n + T], v[b:b + 1, :n + T], 0.4, left, 0, sinks)
            assert np.allclose(O[b], o[0], atol=1e-13) and np.allclose(L[b], l[0], atol=1e-13)
            assert not W[b, :, n + T:].any()
        assert np.allclose(W.sum(2), T * Hq // Hk)


def test_tree_paths_equal_chains():
    """Every path of a tree, alone in the cache, gives its last token the same."""
    parents, T, cap, n = [-1, 0, 0, 1, 1, 2, 4], 7, 16, 5
    words = []
    for t, p in enumerate(parents):
        words.append((words[p] if p >= 0 else 0) | 1 << t)
    q, k, v = _rand(1, 1, T, 2, 4), _rand(2, 1, cap, 1, 4), _rand(3, 1, cap, 1, 4)
    for left, sinks in ((None, 0), (6, 1)):
        O, L, W = oracle.cache_attn(q, k, v, [n], 0.6, [words], left, sinks)
        for t in range(T):
            path = [u for u in range(T) if words[t] >> u & 1]
            rows = list(range(n)) + [n + u for u in path]
            o, l, _ = oracle.cache_attn(q[:, path], k[:, rows], v[:, rows], [n], 0.6, None, left, sinks)
            assert np.allclose(O[0, t], o[0, -1], atol=1e-13) and np.allclose(L[0, :, t], l[0, :, -1], atol=1e-13)
        picked = oracle.cache_attn(q, k, v, [n], 0.6, [words], left, sinks, tokens=[0b10011])[2]
        each = [oracle.cache_attn(q, k, v, [n], 0.6, [words], left, sinks, tokens=[1 << t])[2] for t in (0, 1, 4)]
        assert np.allclose(picked, sum(each), atol=1e-13)


def test_eviction_by_hand():
    w = [5, 1, 3, 3, 0, 3, 9, 2]
    assert oracle.cache_evict(w, 8, 4).tolist() == [0, 2, 3, 6]
    assert oracle.cache_evict(w, 8, 4, 2, 1).tolist() == [0, 1, 6, 7]
    assert oracle.cache_evict(w, 8, 5, 1, 1).tolist() == [0, 2, 3, 6, 7]
    assert oracle.cache_evict(w, 3, 4, 1, 1).tolist() == [0, 1, 2]
    assert oracle.cache_evict(w, 8, 3, 1, 2).tolist() == [0, 6, 7]
    assert oracle.cache_evict([math.nan, -math.inf, math.nan, 0.0, -0.0], 5, 3).tolist() == [1, 3, 4]
    assert oracle.cache_evict([0.0, -0.0, 0.0], 3, 2).tolist() == [0, 1]
