"""Pins of the oracle's rotary positions and cross attention against what the
mathematics fixes (CPU): complex rotations, relative positions, hand-worked
values, central differences, and block-sparse attention where the two meet."""
import numpy as np
import pytest

import oracle


def _pos(rng, rows, axes):
    return rng.integers(0, 50, (rows, axes)) + rng.choice([0.0, 0.5], (rows, axes))


@pytest.mark.parametrize("axes,D", [((4, 6, 6), 16), ((8,), 8), ((2, 4), 12)])
def test_rope_is_a_complex_rotation_in_both_layouts(axes, D):
    rng = np.random.default_rng(1)
    n, H, R = 7, 2, sum(axes)
    x, pos = rng.standard_normal((n, H, D)), _pos(rng, 5, len(axes))
    idx = rng.integers(0, 5, n)
    unit = np.concatenate([np.exp(1j * pos[idx, a][:, None] * 100.0 ** (-np.arange(0, d, 2) / d))
                           for a, d in enumerate(axes)], 1)[:, None]
    near = oracle.rope_fwd(x, pos, axes, 100.0, idx)
    z = (x[..., 0:R:2] + 1j * x[..., 1:R:2]) * unit
    assert np.allclose(near[..., 0:R:2], z.real) and np.allclose(near[..., 1:R:2], z.imag)
    far = oracle.rope_fwd(x, pos, axes, 100.0, idx, interleaved=False)
    z = (x[..., :R // 2] + 1j * x[..., R // 2:R]) * unit
    assert np.allclose(far[..., :R // 2], z.real) and np.allclose(far[..., R // 2:R], z.imag)
    assert np.array_equal(near[..., R:], x[..., R:]) and np.array_equal(far[..., R:], x[..., R:])


def test_rope_scores_depend_on_position_differences_only():
    rng = np.random.default_rng(2)
    q, k = rng.standard_normal((2, 1, 1, 12))
    turn = lambda x, p: oracle.rope_fwd(x, [p], (4, 4, 4), 50.0)[0, 0]  # noqa: E731
    a = turn(q, (3, 10, 7)) @ turn(k, (1, 4, 9))
    b = turn(q, (13, 110, 0.5)) @ turn(k, (11, 104, 2.5))
    assert abs(a - b) < 1e-12
    assert np.allclose(turn(q, (0, 0, 0)), q[0, 0])
    out = oracle.rope_fwd(np.repeat(q, 3, 0), [(1, 2, 3)], (4, 4, 4), 50.0, token_idx=[0, -1, 1])
    assert not np.allclose(out[0], q[0]) and np.allclose(out[1:], q[0])


def test_rope_norm_by_hand():
    # mean square of (3, 4, 0, 0) is 25 / 4; a quarter turn takes (u, v) to (-v, u)
    y = oracle.rope_fwd(np.array([[[3.0, 4.0, 0.0, 0.0]]]), [[np.pi / 2]], (2,), 10.0, weight=[1.0, 2.0, 1.0, 1.0],
                        eps=0.0)
    assert np.allclose(y[0, 0], [-3.2, 1.2, 0.0, 0.0])


@pytest.mark.parametrize("interleaved", [True, False])
def test_rope_gradients_match_central_differences(interleaved):
    rng = np.random.default_rng(3)
    n, H, D, axes = 3, 2, 16, (4, 4)
    x, w, dy = rng.standard_normal((n, H, D)), 1 + 0.3 * rng.standard_normal(D), rng.standard_normal((n, H, D))
    pos = _pos(rng, 2, 2)
    f = lambda a, b: float((oracle.rope_fwd(a, pos, axes, 30.0, weight=b, eps=1e-3,  # noqa: E731
                                            interleaved=interleaved) * dy).sum())
    dx, dw = oracle.rope_bwd(dy, pos, axes, 30.0, x=x, weight=w, eps=1e-3, interleaved=interleaved)
    h = 1e-5
    for _ in range(12):
        i = tuple(rng.integers(0, s) for s in x.shape)
        e = np.zeros_like(x)
        e[i] = h
        assert abs((f(x + e, w) - f(x - e, w)) / (2 * h) - dx[i]) < 1e-8
    for i in range(D):
        e = np.zeros(D)
        e[i] = h
        assert abs((f(x, w + e) - f(x, w - e)) / (2 * h) - dw[i]) < 1e-8
    back, none = oracle.rope_bwd(oracle.rope_fwd(x, pos, axes, 30.0, interleaved=interleaved), pos, axes, 30.0,
                                 interleaved=interleaved)
    assert none is None and np.allclose(back, x)


def _xcase(seed, B, Nq, Nk, Hq, Hk, D):
    rng = np.random.default_rng(seed)
    q, do = rng.standard_normal((2, B, Nq, Hq, D))
    k, v = rng.standard_normal((2, B, Nk, Hk, D))
    return q, k, v, do, rng


def test_xattn_equals_dense_block_sparse_attention_on_equal_lengths():
    q, k, v, do, _ = _xcase(4, 2, 20, 20, 3, 3, 8)
    ones = np.ones((2, 3, 2, 2), np.uint8)
    for a, b in zip(oracle.xattn_fwd(q, k, v, 0.3), oracle.bsattn_fwd(q, k, v, ones, 16, 0.3)):
        assert np.allclose(a, b)
    for a, b in zip(oracle.xattn_bwd(q, k, v, do, 0.3), oracle.bsattn_bwd(q, k, v, do, ones, 16, 0.3)):
        assert np.allclose(a, b)


def test_xattn_by_hand_and_empty_rows():
    q = np.array([1.0, 0.0]).reshape(1, 1, 1, 2)
    k = np.array([[np.log(3.0), 5.0], [0.0, 7.0], [9.0, 9.0]]).reshape(1, 3, 1, 2)
    v = np.array([[4.0, 0.0], [0.0, 8.0], [np.nan, np.inf]]).reshape(1, 3, 1, 2)
    O, L = oracle.xattn_fwd(q, k, v, 1.0, [[1, 1, 0]])
    assert np.allclose(O.ravel(), [3.0, 2.0]) and np.allclose(L.ravel(), np.log(4.0))
    O, L = oracle.xattn_fwd(q, k, v, 1.0, [[0, 0, 0]])
    assert np.all(O == 0) and np.all(L == -np.inf)
    for g in oracle.xattn_bwd(q, k, v, np.ones_like(q), 1.0, [[0, 0, 0]]):
        assert np.all(g == 0)


def test_xattn_gradients_match_central_differences():
    q, k, v, do, rng = _xcase(5, 2, 3, 5, 4, 2, 6)
    mask = np.array([[1, 0, 1, 1, 0], [1, 1, 1, 1, 1]])
    f = lambda a, b, c: float((oracle.xattn_fwd(a, b, c, 0.4, mask)[0] * do).sum())  # noqa: E731
    grads = oracle.xattn_bwd(q, k, v, do, 0.4, mask)
    h = 1e-5
    for t in range(3):
        for _ in range(10):
            x = [q.copy(), k.copy(), v.copy()]
            i = tuple(rng.integers(0, s) for s in x[t].shape)
            x[t][i] += h
            up = f(*x)
            x[t][i] -= 2 * h
            assert abs((up - f(*x)) / (2 * h) - grads[t][i]) < 1e-8
    assert np.all(grads[1][0, [1, 4]] == 0) and np.all(grads[2][0, [1, 4]] == 0)
