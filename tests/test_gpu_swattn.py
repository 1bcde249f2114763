"""Window attention on the GPU against the float64 oracle.

Tolerances: the arithmetic is that of the cross-attention kernels (bf16 products
with fp32 sums, P and dS rounded to bf16 before their second products, outputs
rounded to bf16), so the bounds are theirs. With u = 2^-8 (half a bf16 step), e =
2^-24 and A_ij = sum_d |q_id k_jd| scale, worst cases over the sums:
  scores      d_ij = 2 (D + 8) e A_ij, and 2^-18 for the exponential and the
              conversion to base 2 (|score| up to 40): x = max d_ij + 2^-18
              relative on P before and after normalisation: e_P = 2 x
  LSE         x + 2^-22 max(1, |LSE|)
  O           (u + e_P) sum_j P_ij |v_j| + u |O|
  dV          (u + e_P) sum_i P_ij |dO_i| + u |dV|
  dS          t_ij = (u + e_P) |dS_ij| + P_ij (2 D e sum|dO v| + sum_d |dO_id| tol_O_id)
              (delta is formed from the stored bf16 O)
  dQ, dK      scale sum t |k|, scale sum t |q|, and u |result|
2-norms of the errors: 1e-2 of O and 2e-2 of the gradients (at most four roundings
of relative size u / sqrt(3) each, 9e-3), for windows of several keys; rows that see
one or two keys have gradients of rounding size, held by the element bounds."""
import math

import numpy as np
import pytest
import torch

import oracle
import paper_2609_23169_amd as ut

pytestmark = pytest.mark.gpu
DEV = "cuda"
U, E24 = 2.0 ** -8, 2.0 ** -24


def f64(t):
    return t.detach().double().cpu().numpy()


def check_head(Q, K, V, see, scale, O, L, o, l, label, D):
    """One head's forward results o, l against O, L: (P, x, tolerance of O)."""
    K, V = (np.where(see.any(0)[:, None], x, 0.0) for x in (K, V))
    P, _ = oracle._seen_p(Q, K, scale, see)
    some = see.any(1)
    x = float((np.abs(Q) @ np.abs(K).T).max(initial=0.0)) * scale * 2 * (D + 8) * E24 + 2.0 ** -18
    assert np.all(l[~some] == -np.inf) and np.all(o[~some] == 0), label
    tl = x + 2.0 ** -22 * np.maximum(1, np.abs(L[some]))
    assert np.all(np.abs(l[some] - L[some]) <= tl), (label, "LSE")
    to = (U + 2 * x) * (P @ np.abs(V)) + U * np.abs(O)
    err = np.abs(o - O)
    assert np.all(err <= to), (label, "O", float((err / (to + 1e-30)).max()))
    return P, x, to, K, V


def check(q, k, v, do, scale, window, sinks, mask, o, lse, grads=None, label="", norms=True):
    O, L = oracle.swattn_fwd(q, k, v, scale, *window, sinks, mask)
    B, Nq, Hq, D = q.shape
    Nk, G = k.shape[1], Hq // k.shape[2]
    base = oracle.window_see(Nq, Nk, *window, sinks)
    ref = oracle.swattn_bwd(q, k, v, do, scale, *window, sinks, mask) if grads is not None else None
    tdk, tdv = np.zeros(k.shape), np.zeros(k.shape)
    for b in range(B):
        see = base if mask is None else base & mask[b].astype(bool)[None]
        for h in range(Hq):
            P, x, to, K, V = check_head(q[b, :, h], k[b, :, h // G], v[b, :, h // G], see, scale, O[b, :, h], L[b, h],
                                        o[b, :, h], lse[b, h], label, D)
            if grads is None:
                continue
            dO, Q = do[b, :, h], q[b, :, h]
            dS = P * (dO @ V.T - (dO * O[b, :, h]).sum(1, keepdims=True))
            t = (U + 2 * x) * np.abs(dS) + P * (2 * D * E24 * (np.abs(dO) @ np.abs(V).T)
                                                + (np.abs(dO) * to).sum(1, keepdims=True))
            tq = scale * (t @ np.abs(K)) + U * np.abs(ref[0][b, :, h])
            err = np.abs(grads[0][b, :, h] - ref[0][b, :, h])
            assert np.all(err <= tq + 1e-30), (label, "dQ", float((err / (tq + 1e-30)).max()))
            tdk[b, :, h // G] += scale * (t.T @ np.abs(Q))
            tdv[b, :, h // G] += (U + 2 * x) * (P.T @ np.abs(dO))
    if norms:
        assert np.linalg.norm(o - O) <= 1e-2 * np.linalg.norm(O) + 1e-30, label
    if grads is not None:
        for got, r, t, nm in ((grads[1], ref[1], tdk, "dK"), (grads[2], ref[2], tdv, "dV")):
            t = t + U * np.abs(r)
            err = np.abs(got - r)
            assert np.all(err <= t + 1e-30), (label, nm, float((err / (t + 1e-30)).max()))
        if norms:
            for got, r in zip(grads, ref):
                assert np.linalg.norm(got - r) <= 2e-2 * np.linalg.norm(r) + 1e-30, label


def draw(seed, B, Nq, Nk, Hq, Hk, D, fused=False):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g).to(torch.bfloat16).to(DEV)  # noqa: E731
    q, do = r(B, Nq, Hq, D), r(B, Nq, Hq, D)
    if fused:
        kv = r(B, Nk, 2, Hk, D)
        return q, kv[:, :, 0], kv[:, :, 1], do
    return q, r(B, Nk, Hk, D), r(B, Nk, Hk, D), do


def run(q, k, v, do, scale, window, sinks=0, mask=None, **kw):
    m = None if mask is None else torch.from_numpy(mask).to(DEV)
    o, lse = ut.swattn_fwd(q, k, v, window, scale, sinks, key_mask=m, **kw)
    grads = ut.swattn_bwd(q, k, v, o, do, lse, window, scale, sinks, key_mask=m, **kw)
    torch.cuda.synchronize()
    return o, lse, grads


def random_mask(seed, B, Nk, share=0.6):
    rng = np.random.default_rng(seed)
    return ((rng.random((B, Nk)) < share) * rng.integers(1, 256, (B, Nk))).astype(np.uint8)


def check_case(seed, B, Nq, Nk, Hq, Hk, D, window, sinks, mask=None, fused=False, norms=True):
    q, k, v, do = draw(seed, B, Nq, Nk, Hq, Hk, D, fused)
    o, lse, grads = run(q, k, v, do, D ** -0.5, window, sinks, mask)
    check(*(f64(t) for t in (q, k, v, do)), D ** -0.5, window, sinks, mask, f64(o), f64(lse), [f64(t) for t in grads],
          f"{(B, Nq, Nk, Hq, Hk, D, window, sinks, mask is not None)}", norms)


SHAPES = [  # B, Nq, Nk, Hq, Hk, D, window, sinks
    (1, 1, 1, 1, 1, 64, (0, 0), 0), (1, 1, 1, 1, 1, 8, (5, 0), 1), (2, 65, 65, 2, 1, 128, (16, 0), 0),
    (1, 300, 300, 2, 2, 64, (31, 0), 4), (1, 384, 384, 2, 2, 64, (95, 0), 4), (1, 257, 257, 3, 3, 128, (64, 0), 1),
    (2, 500, 500, 4, 2, 40, (100, 17), 3), (1, 700, 700, 2, 1, 128, (128, 128), 77), (1, 130, 130, 6, 2, 72, (None, 0), 0),
    (1, 200, 200, 2, 2, 128, (None, None), 0), (1, 333, 333, 5, 1, 96, (63, 1), 65), (1, 640, 640, 1, 1, 64, (20, None), 2),
    (1, 1000, 1000, 2, 1, 64, (40, 0), 130), (3, 129, 129, 2, 2, 16, (33, 40), 200), (1, 800, 800, 2, 2, 128, (64, 0), 1),
]


@pytest.mark.parametrize("B,Nq,Nk,Hq,Hk,D,window,sinks", SHAPES)
def test_matches_oracle(B, Nq, Nk, Hq, Hk, D, window, sinks):
    norms = min(Nk, 1 + sum(100 if w is None else w for w in window)) > 4
    check_case(1, B, Nq, Nk, Hq, Hk, D, window, sinks, norms=norms)
    check_case(2, B, Nq, Nk, Hq, Hk, D, window, sinks, random_mask(3, B, Nk), True, norms=norms)


@pytest.mark.parametrize("window,sinks", [((0, 0), 0), ((0, 0), 1), ((1, 0), 0), ((0, 1), 2), ((2, 1), 0)])
@pytest.mark.parametrize("D", [64, 128])
def test_tiny_windows(D, window, sinks):
    check_case(4, 1, 200, 200, 2, 1, D, window, sinks, norms=False)


# queries at the end of more keys, and in front of fewer
@pytest.mark.parametrize("B,Nq,Nk,Hq,Hk,D,window,sinks", [
    (1, 1, 5000, 2, 2, 128, (None, 0), 0), (2, 1, 4099, 8, 2, 64, (1500, 0), 4), (1, 40, 3000, 3, 1, 96, (2000, 0), 70),
    (1, 100, 4100, 2, 2, 128, (300, 0), 4), (1, 64, 700, 4, 2, 64, (100, 50), 1), (1, 300, 100, 2, 1, 64, (40, 0), 2),
    (2, 200, 17, 2, 2, 128, (5, 3), 2), (1, 90, 40, 1, 1, 64, (30, 0), 0), (1, 500, 1, 2, 2, 64, (3, 0), 1),
    (1, 33, 9000, 33, 1, 128, (None, 0), 0), (1, 1, 300, 4, 1, 64, (10, 0), 0),
])
def test_queries_at_the_end_of_the_keys(B, Nq, Nk, Hq, Hk, D, window, sinks):
    check_case(5, B, Nq, Nk, Hq, Hk, D, window, sinks)
    check_case(6, B, Nq, Nk, Hq, Hk, D, window, sinks, random_mask(7, B, Nk, 0.3))


@pytest.mark.parametrize("kind", ["none", "sinks", "tail", "one"])
def test_masks_that_leave_rows_empty(kind):
    B, N = 2, 400
    mask = np.zeros((B, N), np.uint8)
    if kind == "sinks":
        mask[:, :3] = 1
    elif kind == "tail":
        mask[:, 350:] = 9
    elif kind == "one":
        mask[0, 200] = 255
    for window, sinks in (((50, 0), 4), ((30, 30), 2), ((50, 0), 0)):
        check_case(8, B, N, N, 4, 2, 64, window, sinks, mask, norms=False)


def test_sinks_that_a_long_sequence_sees():
    """Partial sums for the keys in the sinks' tiles, whole ones for the others."""
    for D, window, sinks, Hq, Hk in ((64, (40, 0), 4, 2, 1), (128, (30, 20), 150, 1, 1), (128, (200, 0), 1, 3, 3)):
        assert ut.ut_swattn_bwd_workspace_size(1, 4000, 4000, Hq, Hk, D, window, sinks) > \
            ut.ut_swattn_bwd_workspace_size(1, 4000, 4000, Hq, Hk, D, window, 0)
        check_case(9, 1, 4000, 4000, Hq, Hk, D, window, sinks)


@pytest.mark.parametrize("n,Hq,Hk,D,window,sinks", [(2, 24, 24, 80, (17, 17), 4), (40, 4, 2, 64, (9, 0), 2), (64, 3, 3, 128, (63, 63), 0)])
def test_small_grids_round_ds_once_less(n, Hq, Hk, D, window, sinks):
    """dS goes into its products with what its rounding left: its error is 2^-16 of it (two
    half steps of bf16, 2^-8 each) in place of 2^-8, so that dQ and dK are off by their
    own rounding and little else. One tile of keys: delta is formed in fp32."""
    q, k, v, do = draw(40 + n, 2, n, n, Hq, Hk, D)
    scale = D ** -0.5
    _, _, grads = run(q, k, v, do, scale, window, sinks)
    Q, K, V, dO = f64(q), f64(k), f64(v), f64(do)
    ref = oracle.swattn_bwd(Q, K, V, dO, scale, *window, sinks, None)
    see, G = oracle.window_see(n, n, *window, sinks), Hq // Hk
    tdk = np.zeros(K.shape)
    for b in range(2):
        for h in range(Hq):
            qh, kh, vh, dh = Q[b, :, h], K[b, :, h // G], V[b, :, h // G], dO[b, :, h]
            P, _ = oracle._seen_p(qh, kh, scale, see)
            x = float((np.abs(qh) @ np.abs(kh).T).max()) * scale * 2 * (D + 8) * E24 + 2.0 ** -18
            dP = dh @ vh.T
            dS = P * (dP - (P * dP).sum(1, keepdims=True))
            wide = np.abs(dh) @ np.abs(vh).T
            t = (2.0 ** -16 + 2 * x) * np.abs(dS) + P * ((2 * D * E24 + 2 * x) * (wide + (P * wide).sum(1, keepdims=True)))
            tq = scale * (t @ np.abs(kh)) + U * np.abs(ref[0][b, :, h])
            assert np.all(np.abs(f64(grads[0])[b, :, h] - ref[0][b, :, h]) <= tq + 1e-30)
            tdk[b, :, h // G] += scale * (t.T @ np.abs(qh))
    assert np.all(np.abs(f64(grads[1]) - ref[1]) <= tdk + U * np.abs(ref[1]) + 1e-30)


def test_seeded_sweep():
    rng = np.random.default_rng(12)
    for i in range(30):
        Hk = int(rng.choice([1, 2, 3]))
        Nq = int(round(math.exp(rng.uniform(0, math.log(900)))))
        Nk = Nq if i % 3 else int(round(math.exp(rng.uniform(0, math.log(1500)))))
        B = int(rng.integers(1, 4))
        left = [None, int(rng.integers(8, 500))][int(rng.random() < 0.8)]
        right = [0, 0, int(rng.integers(1, 300)), None][int(rng.integers(0, 4))]
        check_case(100 + i, B, Nq, Nk, Hk * int(rng.choice([1, 2, 5])), Hk, 8 * int(rng.integers(1, 17)), (left, right),
                   int(rng.choice([0, 1, 4, 64, 100])), random_mask(i, B, Nk) if rng.random() < 0.4 else None,
                   bool(rng.integers(0, 2)), norms=Nk > 8)


@pytest.mark.parametrize("Nq,Nk", [(1, 5), (7, 64), (300, 300), (1000, 77), (1, 5000)])
@pytest.mark.parametrize("D", [64, 128])
def test_no_bounds_is_cross_attention(Nq, Nk, D):
    q, k, v, do = draw(10, 2, Nq, Nk, 4, 2, D)
    mask = random_mask(11, 2, Nk)
    m = torch.from_numpy(mask).to(DEV)
    o, lse, grads = run(q, k, v, do, 0.1, (None, None), 3, mask)
    o2, lse2 = ut.xattn_fwd(q, k, v, 0.1, key_mask=m)
    grads2 = ut.xattn_bwd(q, k, v, o2, do, lse2, 0.1, key_mask=m)
    for x, y in zip((o, lse) + grads, (o2, lse2) + grads2):
        assert torch.allclose(x.float(), y.float(), rtol=2 ** -6, atol=2 ** -6)
    assert torch.equal(o, o2) and torch.equal(lse, lse2)


def test_equal_results_on_every_run():
    q, k, v, do = draw(13, 2, 900, 900, 4, 2, 128)
    a, b = (run(q, k, v, do, 0.1, (100, 0), 4) for _ in range(2))
    for x, y in zip((a[0], a[1]) + a[2], (b[0], b[1]) + b[2]):
        assert torch.equal(x, y)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -3.3e38])
def test_keys_that_no_query_sees_may_hold_anything(bad):
    """Unused by the mask, and out of every window (more keys than reach)."""
    q, k, v, do = draw(14, 2, 60, 500, 4, 2, 128)
    mask = random_mask(15, 2, 500)
    seen = oracle.window_see(60, 500, 100, 0, 2).any(0)[None] & (mask != 0)
    a = run(q, k, v, do, 0.09, (100, 0), 2, mask)
    off = torch.from_numpy(~seen).to(DEV)
    k2, v2 = k.clone(), v.clone()
    k2[off], v2[off] = bad, bad
    b = run(q, k2, v2, do, 0.09, (100, 0), 2, mask)
    for x, y in zip((a[0], a[1]) + a[2], (b[0], b[1]) + b[2]):
        assert torch.equal(x, y)
    assert (b[2][1][off] == 0).all() and (b[2][2][off] == 0).all()


def test_a_far_outlier_does_not_reach_windows_without_it():
    """One key of huge score: rows that do not see it keep their results to the bit."""
    q, k, v, do = draw(16, 1, 600, 600, 2, 2, 64)
    want = run(q, k, v, do, 0.125, (64, 0), 0)
    k2 = k.clone()
    k2[0, 200] *= 100
    got = run(q, k2, v, do, 0.125, (64, 0), 0)
    rows = torch.ones(600, dtype=torch.bool, device=DEV)
    rows[200:265] = False
    assert torch.equal(got[0][:, rows], want[0][:, rows]) and torch.equal(got[1][:, :, rows], want[1][:, :, rows])
    assert torch.equal(got[2][0][:, rows], want[2][0][:, rows])


def test_scores_far_apart():
    q, k, v, do = draw(17, 1, 400, 400, 2, 2, 64)
    k = k * torch.linspace(0.1, 6, 400, device=DEV)[None, :, None, None].to(torch.bfloat16)
    for scale in (0.125, 2.0):
        o, lse = ut.swattn_fwd(q, k, v, (70, 0), scale, 3)
        O, L = oracle.swattn_fwd(f64(q), f64(k), f64(v), scale, 70, 0, 3)
        x = scale * float((np.abs(f64(q)[0, :, 0]) @ np.abs(f64(k)[0, :, 0]).T).max()) * 2 * 72 * E24 + 2.0 ** -18
        assert np.all(np.abs(f64(lse) - L) <= x + 2.0 ** -22 * np.maximum(1, np.abs(L)))
        assert np.abs(f64(o) - O).max() <= (2 * U + 4 * x) * np.abs(f64(v)).max()


def test_strided_views_in_and_out():
    B, N, Hq, Hk, D, window, sinks = 2, 390, 4, 2, 64, (50, 20), 5
    q, k, v, do = draw(18, B, N, N, Hq, Hk, D)
    o, lse, grads = run(q, k, v, do, 0.125, window, sinks)
    big = torch.full((B, N, 5, Hq, D), 3.0, dtype=torch.bfloat16, device=DEV)
    kv = torch.full((B, N, 5, Hk, D), 3.0, dtype=torch.bfloat16, device=DEV)
    big[:, :, 0], big[:, :, 2], kv[:, :, 0], kv[:, :, 1] = q, do, k, v
    l2 = torch.empty_like(lse)
    assert ut.ut_swattn_fwd(big[:, :, 0], kv[:, :, 0], kv[:, :, 1], big[:, :, 1], l2, window, 0.125, sinks) == ut.UT_OK
    ws = torch.empty(ut.ut_swattn_bwd_workspace_size(B, N, N, Hq, Hk, D, window, sinks), dtype=torch.uint8, device=DEV)
    assert ut.ut_swattn_bwd(big[:, :, 0], kv[:, :, 0], kv[:, :, 1], big[:, :, 1], big[:, :, 2], l2, big[:, :, 3],
                            kv[:, :, 2], kv[:, :, 3], window, 0.125, sinks, workspace=ws) == ut.UT_OK
    for x, y in ((big[:, :, 1], o), (l2, lse), (big[:, :, 3], grads[0]), (kv[:, :, 2], grads[1]), (kv[:, :, 3], grads[2])):
        assert torch.equal(x, y)
    assert (big[:, :, 4] == 3).all() and (kv[:, :, 4] == 3).all()


def test_workspace_of_any_content():
    q, k, v, do = draw(19, 1, 3000, 3000, 2, 2, 64)
    window, sinks = (40, 0), 4
    want = run(q, k, v, do, 0.125, window, sinks)
    size = ut.ut_swattn_bwd_workspace_size(1, 3000, 3000, 2, 2, 64, window, sinks)
    guard = torch.full((size + 4096,), 0xFF, dtype=torch.uint8, device=DEV)
    got = ut.swattn_bwd(q, k, v, want[0], do, want[1], window, 0.125, sinks, workspace=guard[:size])
    for x, y in zip(got, want[2]):
        assert torch.equal(x, y)
    assert (guard[size:] == 0xFF).all()


def test_zero_lengths():
    q, k, v, do = draw(20, 2, 5, 0, 2, 1, 64)
    o, lse, (dq, dk, dv) = run(q, k, v, do, 0.125, (3, 0), 2)
    assert (o == 0).all() and (lse == -math.inf).all() and (dq == 0).all() and dk.shape == k.shape
    q, k, v, do = draw(20, 2, 0, 70, 2, 1, 64)
    o, lse, (dq, dk, dv) = run(q, k, v, do, 0.125, (3, 0), 2)
    assert o.numel() == 0 and dq.numel() == 0 and (dk == 0).all() and (dv == 0).all()


def test_keys_past_32_bit_offsets():
    Nk, stride, H, D = 600, (1 << 22) - 8, 1, 64
    q, k, v, do = draw(21, 1, 50, Nk, H, H, D)
    buf = torch.empty((Nk - 1) * stride + 2 * D, dtype=torch.bfloat16, device=DEV)
    kf = torch.as_strided(buf, (1, Nk, H, D), (Nk * stride, stride, D, 1))
    vf = torch.as_strided(buf, (1, Nk, H, D), (Nk * stride, stride, D, 1), D)
    kf.copy_(k), vf.copy_(v)
    a, b = (run(q, *x, do, 0.125, (100, 0), 70) for x in ((k, v), (kf, vf)))
    for x, y in zip((a[0], a[1]) + a[2], (b[0], b[1]) + b[2]):
        assert torch.equal(x, y)


# ---- packed samples --------------------------------------------------------

def offsets(lens):
    return torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device=DEV)


VARLEN = [  # lq, lk, Hq, Hk, D, window, sinks
    ([70, 130, 1, 333], [70, 130, 1, 333], 4, 2, 64, (40, 0), 3), ([5, 0, 300], [0, 77, 300], 2, 2, 128, (64, 30), 70),
    ([1] * 6, [700] * 6, 8, 2, 128, (500, 0), 4), ([200], [300], 3, 1, 72, (None, 0), 0),
    ([0, 0, 40], [50, 0, 9], 2, 1, 40, (6, 2), 1), ([1, 2, 3], [4200, 1, 9000], 4, 1, 64, (None, 0), 2),
    ([2100, 1800], [2100, 1800], 2, 2, 128, (30, 0), 2),
]


@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("lq,lk,Hq,Hk,D,window,sinks", VARLEN)
def test_varlen_matches_oracle(lq, lk, Hq, Hk, D, window, sinks, masked):
    rest, g = 13, torch.Generator().manual_seed(22)
    r = lambda n, h: torch.randn((n, h, D), generator=g).to(torch.bfloat16).to(DEV)  # noqa: E731
    Tq, Tk, scale = sum(lq) + rest, sum(lk) + rest, D ** -0.5
    q, do, k, v = r(Tq, Hq), r(Tq, Hq), r(Tk, Hk), r(Tk, Hk)
    mask = random_mask(23, 1, Tk)[0] if masked else None
    m = None if mask is None else torch.from_numpy(mask).to(DEV)
    at = (offsets(lq), max(lq), offsets(lk), max(lk), window)
    o, lse = ut.swattn_fwd_varlen(q, k, v, *at, scale, sinks, key_mask=m)
    grads = ut.swattn_bwd_varlen(q, k, v, o, do, lse, *at, scale, sinks, key_mask=m)
    torch.cuda.synchronize()
    eq, ek = np.concatenate([[0], np.cumsum(lq)]), np.concatenate([[0], np.cumsum(lk)])
    for b in range(len(lq)):
        sq, sk = slice(eq[b], eq[b + 1]), slice(ek[b], ek[b + 1])
        check(*(f64(x[s])[None] for x, s in ((q, sq), (k, sk), (v, sk), (do, sq))), scale, window, sinks,
              None if mask is None else mask[sk][None], f64(o[sq])[None], f64(lse[:, sq])[None],
              [f64(x[s])[None] for x, s in zip(grads, (sq, sk, sk))], f"sample {b}", norms=False)
    for x, n in ((o, sum(lq)), (grads[0], sum(lq)), (grads[1], sum(lk)), (grads[2], sum(lk))):
        assert (x[n:] == 0).all()
    assert (lse[:, sum(lq):] == -math.inf).all()


def test_varlen_rows_behind_the_last_sample_stay():
    lens, T, H, D, window = [300, 200], 600, 2, 64, (30, 0)
    g = torch.Generator().manual_seed(24)
    q, k, v, do = (torch.randn((T, H, D), generator=g).to(torch.bfloat16).to(DEV) for _ in range(4))
    at = (offsets(lens), 300, offsets(lens), 300, window)
    o, lse = torch.full_like(q, 7), torch.full((H, T), 7.0, device=DEV)
    dq, dk, dv = (torch.full_like(q, 7) for _ in range(3))
    assert ut.ut_swattn_fwd_varlen(q, k, v, o, lse, *at, 0.125, 2) == ut.UT_OK
    ws = torch.empty(ut.ut_swattn_bwd_varlen_workspace_size(2, T, T, 300, 300, H, H, D, window, 2), dtype=torch.uint8,
                     device=DEV)
    assert ut.ut_swattn_bwd_varlen(q, k, v, o, do, lse, dq, dk, dv, *at, 0.125, 2, workspace=ws) == ut.UT_OK
    for x in (o, dq, dk, dv):
        assert (x[500:] == 7).all() and not (x[:500] == 7).all()
    assert (lse[:, 500:] == 7).all()


def test_varlen_bad_offsets_write_nothing_outside():
    """Offsets are clamped in the kernels: whatever they hold, what lies around the
    buffers stays."""
    T, H, D, window = 200, 2, 64, (20, 5)
    bufs = [torch.full((T + 64, H, D), 3.0, dtype=torch.bfloat16, device=DEV) for _ in range(8)]
    q, k, v, o, do, dq, dk, dv = (b[32:32 + T] for b in bufs)
    lse = torch.zeros((H, T), device=DEV)
    ws = torch.empty(ut.ut_swattn_bwd_varlen_workspace_size(2, T, T, 150, 150, H, H, D, window, 3) + 16, dtype=torch.uint8,
                     device=DEV)
    for cu in ([0, 150, 5000], [0, -7, 100], [190, 20, 210], [-5, 199, 300]):
        c = torch.tensor(cu, dtype=torch.int32, device=DEV)
        assert ut.ut_swattn_fwd_varlen(q, k, v, o, lse, c, 150, c, 150, window, 0.125, 3, None, True) == ut.UT_OK
        assert ut.ut_swattn_bwd_varlen(q, k, v, o, do, lse, dq, dk, dv, c, 150, c, 150, window, 0.125, 3, None, True,
                                       ws) == ut.UT_OK
    torch.cuda.synchronize()
    for b in bufs:
        assert (b[:32] == 3).all() and (b[32 + T:] == 3).all()


# ---- streams, graphs -------------------------------------------------------

def test_on_another_stream_and_captured():
    q, k, v, do = draw(25, 1, 2500, 2500, 4, 2, 64)
    window, sinks = (60, 0), 4
    want = run(q, k, v, do, 0.125, window, sinks)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    o, lse = ut.swattn_fwd(q, k, v, window, 0.125, sinks, stream=s)
    grads = ut.swattn_bwd(q, k, v, o, do, lse, window, 0.125, sinks, stream=s)
    s.synchronize()
    for x, y in zip((o, lse) + grads, (want[0], want[1]) + want[2]):
        assert torch.equal(x, y)
    graph = torch.cuda.CUDAGraph()
    q2 = q.clone()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        o, lse = ut.swattn_fwd(q2, k, v, window, 0.125, sinks)
        grads = ut.swattn_bwd(q2, k, v, o, do, lse, window, 0.125, sinks)
    for turn in range(3):
        q2.copy_(q if turn != 1 else -q)
        graph.replay()
        ref = run(q2, k, v, do, 0.125, window, sinks)
        torch.cuda.synchronize()
        for x, y in zip((o, lse) + grads, (ref[0], ref[1]) + ref[2]):
            assert torch.equal(x, y)
