"""Gradients of window attention where rows see few keys. There dP - delta is a small
difference, and a delta formed from the rounded O that is stored would show in it: rows
that see 16 keys or fewer have it from P and dP in fp32, wherever their keys lie.

Tolerances. A value rounded to bf16 is off by a share of itself that is even within half
a step, 2^-8 of its power of two at most: 2^-7 / sqrt(12) rms of that power, and over
mantissas m in [1, 2) spread evenly in their logarithm sqrt(mean of 1 / m^2) = sqrt(3 /
(8 ln 2)) of that, 0.00166. dQ and dK carry two such roundings, dS's and their own, 0.00235
of the norm; the bound is that of three, 0.00287. Elements: as in the other tests of
windows, but delta's part without O's rounding."""
import numpy as np
import pytest
import torch

import oracle
import paper_2609_23169_amd as ut
from test_gpu_swattn import E24, U, check_case, draw, f64, offsets, random_mask, run

pytestmark = pytest.mark.gpu
DEV = "cuda"
THREE = 3 ** 0.5 * 2.0 ** -7 / 12 ** 0.5 * (3 / (8 * np.log(2))) ** 0.5


def check_exact_delta(q, k, v, do, scale, window, sinks, grads, mask=None, norms=True, rows=slice(None)):
    """All rows of `rows` see so few keys."""
    Q, K, V, dO = f64(q), f64(k), f64(v), f64(do)
    ref = oracle.swattn_bwd(Q, K, V, dO, scale, *window, sinks, mask)
    B, n, Hq, D = Q.shape
    base, G = oracle.window_see(n, K.shape[1], *window, sinks), Hq // K.shape[2]
    for b in range(B):
        see = base if mask is None else base & (mask[b] != 0)[None]
        for h in range(Hq):
            qh, kh, vh, dh = Q[b, :, h], K[b, :, h // G], V[b, :, h // G], dO[b, :, h]
            P, _ = oracle._seen_p(qh, kh, scale, see)
            x = float((np.abs(qh) @ np.abs(kh).T).max()) * scale * 2 * (D + 8) * E24 + 2.0 ** -18
            dP = dh @ vh.T
            dS = P * (dP - (P * dP).sum(1, keepdims=True))
            wide = np.abs(dh) @ np.abs(vh).T
            t = (U + 2 * x) * np.abs(dS) + P * ((2 * D * E24 + 2 * x) * (wide + (P * wide).sum(1, keepdims=True)))
            tq = scale * (t @ np.abs(kh)) + U * np.abs(ref[0][b, :, h])
            err = np.abs(f64(grads[0])[b, :, h] - ref[0][b, :, h])
            assert np.all(err[rows] <= tq[rows] + 1e-30), (b, h, float((err / (tq + 1e-30))[rows].max()))
    if norms:
        for got, r in zip(grads[:2], ref):
            off = np.linalg.norm(f64(got) - r) / np.linalg.norm(r)
            assert off <= THREE, off


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("window,sinks", [((1, 0), 0), ((0, 1), 0), ((2, 0), 0), ((2, 1), 0), ((7, 0), 1), ((4, 4), 7), ((0, 0), 1)])
def test_rows_of_few_keys_in_a_long_sequence(D, window, sinks):
    n, H, scale = 2048, 10, D ** -0.5
    q, k, v, do = draw(60, 1, n, n, H, H, D)
    _, _, grads = run(q, k, v, do, scale, window, sinks)
    check_exact_delta(q, k, v, do, scale, window, sinks, grads)


@pytest.mark.parametrize("B,Nq,Nk,Hq,Hk,D,window,sinks", [
    (1, 700, 700, 4, 2, 72, (5, 0), 9), (2, 300, 500, 6, 2, 64, (3, 4), 2), (1, 500, 300, 3, 1, 128, (2, 1), 3),
    (1, 40, 900, 33, 1, 128, (10, 0), 2), (3, 1, 400, 8, 2, 40, (1, 0), 5), (1, 900, 900, 5, 5, 96, (1 << 20, 0), 0),
])
def test_few_keys_match_oracle(B, Nq, Nk, Hq, Hk, D, window, sinks):
    """Shared key heads, queries in front of and behind the keys, starts of a sequence whose
    later rows see much."""
    check_case(61, B, Nq, Nk, Hq, Hk, D, window, sinks, norms=False)
    check_case(62, B, Nq, Nk, Hq, Hk, D, window, sinks, random_mask(63, B, Nk), True, norms=False)
    q, k, v, do = draw(64, B, Nq, Nk, Hq, Hk, D)
    mask = random_mask(65, B, Nk)
    few = np.arange(Nq) + Nk - Nq < 16 if window[0] > 1000 else slice(None)
    for m in (None, mask):
        _, _, grads = run(q, k, v, do, D ** -0.5, window, sinks, m)
        check_exact_delta(q, k, v, do, D ** -0.5, window, sinks, grads, m, False, few)


def test_split_and_packed_rows():
    lens, H, D, window, scale = [300, 1, 77, 2000], 2, 64, (6, 1), 0.125
    T, at = sum(lens), np.concatenate([[0], np.cumsum(lens)])
    q, k, v, do = (x[0] for x in draw(66, 1, T, T, H, H, D))
    cu = (offsets(lens), max(lens), offsets(lens), max(lens), window)
    o, lse = ut.swattn_fwd_varlen(q, k, v, *cu, scale, 3)
    grads = ut.swattn_bwd_varlen(q, k, v, o, do, lse, *cu, scale, 3)
    for a, z in zip(at, at[1:]):
        check_exact_delta(*(x[a:z][None] for x in (q, k, v, do)), scale, window, 3, [g[a:z][None] for g in grads], None, False)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_keys_that_no_row_sees_stay_out_of_delta(bad):
    q, k, v, do = draw(67, 1, 30, 600, 4, 2, 128)
    mask = random_mask(68, 1, 600)
    seen = oracle.window_see(30, 600, 9, 0, 3).any(0)[None] & (mask != 0)
    want = run(q, k, v, do, 0.09, (9, 0), 3, mask)
    off = torch.from_numpy(~seen).to(DEV)
    k[off], v[off] = bad, bad
    got = run(q, k, v, do, 0.09, (9, 0), 3, mask)
    for x, y in zip((want[0], want[1]) + want[2], (got[0], got[1]) + got[2]):
        assert torch.equal(x, y)
