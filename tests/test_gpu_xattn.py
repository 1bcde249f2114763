"""Cross attention on the GPU against the float64 oracle.

Tolerances. Kernel arithmetic: bf16 products with fp32 sums, P and dS rounded to
bf16 before their second products, outputs rounded to bf16. With u = 2^-8 (half a
bf16 step), e = 2^-24, A_ij = sum_d |q_id k_jd| scale and the bounds worst cases
over the sums:
  scores      d_ij = 2 (D + 8) e A_ij, and 2^-18 for the exponential and the
              conversion to base 2 (|score| up to 40): x = max d_ij + 2^-18
              relative on P before and after normalisation: e_P = 2 x
  LSE         x + 2^-22 max(1, |LSE|)
  O           (u + e_P) sum_j P_ij |v_j| + u |O|
  dV          (u + e_P) sum_i P_ij |dO_i| + u |dV|
  dS          t_ij = (u + e_P) |dS_ij| + P_ij (2 D e sum|dO v| + sum_d |dO_id| tol_O_id)
              (delta is formed from the stored bf16 O)
  dQ, dK      scale sum t |k|, scale sum t |q|, and u |result|
and, since worst cases over long sums are loose, the 2-norms of the errors:
1e-2 of O, 2e-2 of the gradients, as for the block-sparse calls (roundings of
relative size u / sqrt(3) each, at most four of them: 9e-3)."""
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


def fro(a, b):
    return float(np.linalg.norm(a - b) / max(np.linalg.norm(b), 1e-30))


def check(q, k, v, do, scale, mask, o, lse, grads=None, label=""):
    """One sample set in the uniform layout, results and inputs as float64."""
    O, L = oracle.xattn_fwd(q, k, v, scale, mask)
    B, Nq, Hq, D = q.shape
    Nk, G = k.shape[1], Hq // k.shape[2]
    ref = oracle.xattn_bwd(q, k, v, do, scale, mask) if grads is not None else None
    tdk, tdv = np.zeros(k.shape), np.zeros(k.shape)
    for b in range(B):
        used = np.ones(Nk, bool) if mask is None else mask[b].astype(bool)
        for h in range(Hq):
            K, V = (np.where(used[:, None], x[b, :, h // G], 0.0) for x in (k, v))
            Q = q[b, :, h]
            got_l = lse[b, h]
            if not used.any():
                assert np.all(got_l == -np.inf) and np.all(o[b, :, h] == 0), label
                if grads is not None:
                    assert np.all(grads[0][b, :, h] == 0), label
                continue
            P, _ = oracle._xattn_p(Q, K, scale, used)
            x = float((np.abs(Q) @ np.abs(K).T).max(initial=0.0)) * scale * 2 * (D + 8) * E24 + 2.0 ** -18
            tl = x + 2.0 ** -22 * np.maximum(1, np.abs(L[b, h]))
            assert np.all(np.abs(got_l - L[b, h]) <= tl), (label, float((np.abs(got_l - L[b, h]) / tl).max()))
            to = (U + 2 * x) * (P @ np.abs(V)) + U * np.abs(O[b, :, h])
            err = np.abs(o[b, :, h] - O[b, :, h])
            assert np.all(err <= to), (label, "O", float((err / to).max()))
            if grads is None:
                continue
            dO = do[b, :, h]
            dS = P * (dO @ V.T - (dO * O[b, :, h]).sum(1, keepdims=True))
            t = (U + 2 * x) * np.abs(dS) + P * (2 * D * E24 * (np.abs(dO) @ np.abs(V).T)
                                                + (np.abs(dO) * to).sum(1, keepdims=True))
            tq = scale * (t @ np.abs(K)) + U * np.abs(ref[0][b, :, h])
            err = np.abs(grads[0][b, :, h] - ref[0][b, :, h])
            assert np.all(err <= tq + 1e-30), (label, "dQ", float((err / (tq + 1e-30)).max()))
            tdk[b, :, h // G] += scale * (t.T @ np.abs(Q))
            tdv[b, :, h // G] += (U + 2 * x) * (P.T @ np.abs(dO))
    if O.size:
        assert fro(o, O) <= 1e-2, (label, fro(o, O))
    if grads is not None:
        for got, r, t, nm in ((grads[1], ref[1], tdk, "dK"), (grads[2], ref[2], tdv, "dV")):
            t = t + U * np.abs(r)
            err = np.abs(got - r)
            assert np.all(err <= t + 1e-30), (label, nm, float((err / (t + 1e-30)).max()))
        for got, r in zip(grads, ref):
            # rows that see one key have gradients of rounding size alone: nothing to compare them with
            if np.linalg.norm(r) > 1e-6 * np.sqrt(max(r.size, 1)):
                assert np.linalg.norm(got - r) <= 2e-2 * np.linalg.norm(r) + 1e-30, (label, fro(got, r))


def draw(seed, B, Nq, Nk, Hq, Hk, D, fused=False):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g).to(torch.bfloat16).to(DEV)  # noqa: E731
    q, do = r(B, Nq, Hq, D), r(B, Nq, Hq, D)
    if fused:
        kv = r(B, Nk, 2, Hk, D)
        return q, kv[:, :, 0], kv[:, :, 1], do
    return q, r(B, Nk, Hk, D), r(B, Nk, Hk, D), do


def make_mask(kind, B, Nk, seed=0):
    rng = np.random.default_rng(seed)
    if kind is None:
        return None
    m = np.zeros((B, Nk), np.uint8)
    for b in range(B):
        if kind == "random":
            m[b] = (rng.random(Nk) < 0.5) * rng.integers(1, 256, Nk)      # any nonzero byte
        elif kind == "right":
            m[b, :max(0, Nk - b * (Nk // max(B - 1, 1)))] = 1             # the last sample has none
        elif kind == "left":
            m[b, Nk // 2 + b:] = 1
        elif kind == "last":
            m[b, Nk - 1:] = 255
        elif kind == "sparse":
            m[b, rng.integers(0, max(Nk, 1), 3) if Nk else []] = 1
        elif kind == "none":
            pass
    return m


def run(q, k, v, do, scale, mask, **kw):
    m = None if mask is None else torch.from_numpy(mask).to(DEV)
    o, lse = ut.xattn_fwd(q, k, v, scale, key_mask=m, **kw)
    grads = ut.xattn_bwd(q, k, v, o, do, lse, scale, key_mask=m, **kw)
    torch.cuda.synchronize()
    return o, lse, grads


def check_case(seed, B, Nq, Nk, Hq, Hk, D, kind=None, fused=False, scale=None):
    q, k, v, do = draw(seed, B, Nq, Nk, Hq, Hk, D, fused)
    scale = scale or 1 / math.sqrt(D)
    mask = make_mask(kind, B, Nk, seed)
    o, lse, grads = run(q, k, v, do, scale, mask)
    for t in (o,) + tuple(grads):
        assert t.dtype == torch.bfloat16 and t.is_contiguous()
    check(*(f64(t) for t in (q, k, v, do)), scale, mask, f64(o), f64(lse), [f64(t) for t in grads],
          f"{(B, Nq, Nk, Hq, Hk, D, kind)}")


SHAPES = [  # B, Nq, Nk, Hq, Hk, D
    (1, 1, 1, 1, 1, 64), (1, 1, 1, 1, 1, 8), (2, 1, 64, 4, 4, 128), (1, 3, 65, 6, 2, 64), (3, 33, 63, 2, 1, 128),
    (1, 128, 77, 2, 2, 64), (1, 129, 128, 3, 3, 128), (2, 257, 300, 4, 1, 40), (1, 64, 513, 12, 4, 72),
    (1, 500, 129, 5, 1, 96), (2, 31, 200, 3, 3, 120), (1, 1000, 20, 2, 2, 128), (1, 65, 640, 8, 8, 16),
    (4, 17, 1, 2, 1, 128), (1, 200, 191, 7, 7, 80), (1, 400, 256, 2, 2, 56),
]


@pytest.mark.parametrize("B,Nq,Nk,Hq,Hk,D", SHAPES)
def test_matches_oracle(B, Nq, Nk, Hq, Hk, D):
    check_case(1, B, Nq, Nk, Hq, Hk, D)
    check_case(2, B, Nq, Nk, Hq, Hk, D, "random", fused=True)


@pytest.mark.parametrize("kind", ["random", "right", "left", "last", "sparse", "none"])
@pytest.mark.parametrize("B,Nq,Nk,Hq,Hk,D", [(3, 70, 333, 4, 2, 64), (2, 5, 129, 2, 2, 128), (1, 300, 64, 2, 1, 128),
                                             (2, 1, 4200, 4, 1, 64)])
def test_masks(B, Nq, Nk, Hq, Hk, D, kind):
    check_case(3, B, Nq, Nk, Hq, Hk, D, kind)


# few rows and many keys (keys split), many rows and few keys (rows split), more
# than 64 tiles of 64 keys, groups that do not divide 32
@pytest.mark.parametrize("B,Nq,Nk,Hq,Hk,D,kind", [
    (1, 1, 5000, 2, 2, 128, None), (2, 1, 4099, 8, 2, 64, "right"), (1, 4, 9001, 5, 1, 128, "sparse"),
    (1, 40, 3000, 3, 1, 96, None), (1, 3000, 70, 2, 1, 128, "random"), (1, 2500, 300, 1, 1, 64, None),
    (2, 1500, 33, 3, 3, 40, "left"), (1, 7, 1025, 33, 1, 128, None), (1, 100, 12300, 1, 1, 64, "random"),
])
def test_split_work(B, Nq, Nk, Hq, Hk, D, kind):
    check_case(4, B, Nq, Nk, Hq, Hk, D, kind)


def test_seeded_sweep():
    rng = np.random.default_rng(11)
    for i in range(24):
        Hk = int(rng.choice([1, 2, 3]))
        Nq, Nk = (int(round(math.exp(rng.uniform(0, math.log(m))))) for m in (900, 2500))
        check_case(100 + i, int(rng.integers(1, 4)), Nq, Nk, Hk * int(rng.choice([1, 2, 5])), Hk,
                   8 * int(rng.integers(1, 17)), rng.choice([None, "random", "right", "left"]), bool(rng.integers(0, 2)))


def test_peaked_and_large_scores():
    """Scores far apart: the running maximum is replaced after the first tile."""
    q, k, v, do = draw(5, 1, 150, 400, 2, 2, 64)
    k = k * torch.linspace(0.1, 6, 400, device=DEV)[None, :, None, None].to(torch.bfloat16)
    for scale in (0.125, 2.0):
        o, lse = ut.xattn_fwd(q, k, v, scale)
        O, L = oracle.xattn_fwd(f64(q), f64(k), f64(v), scale)
        # scores up to about 1000: 2 (D + 8) e A with A up to 3000, and its exponent's share of O
        x = scale * float((np.abs(f64(q)[0, :, 0]) @ np.abs(f64(k)[0, :, 0]).T).max()) * 2 * 72 * E24 + 2.0 ** -18
        tl = x + 2.0 ** -22 * np.maximum(1, np.abs(L))
        assert np.all(np.abs(f64(lse) - L) <= tl)
        P = np.abs(f64(v)).max()
        assert np.abs(f64(o) - O).max() <= (2 * U + 4 * x) * P


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf"), -3.3e38])
@pytest.mark.parametrize("Nq,Nk", [(40, 200), (1, 4500), (700, 90)])
def test_unused_keys_may_hold_anything(Nq, Nk, bad):
    q, k, v, do = draw(6, 2, Nq, Nk, 4, 2, 128)
    mask = make_mask("random", 2, Nk, 5)
    mask[1, Nk // 2:] = 0
    a = run(q, k, v, do, 0.09, mask)
    off = torch.from_numpy(mask == 0).to(DEV)
    k2, v2 = k.clone(), v.clone()
    k2[off], v2[off] = bad, bad
    b = run(q, k2, v2, do, 0.09, mask)
    for x, y in zip((a[0], a[1]) + a[2], (b[0], b[1]) + b[2]):
        assert torch.equal(x, y)
    assert (b[2][1][off] == 0).all() and (b[2][2][off] == 0).all()


def test_a_bad_query_row_stays_its_own():
    q, k, v, do = draw(14, 1, 200, 150, 4, 2, 128)
    want = run(q, k, v, do, 0.1, None)
    for bad in (float("nan"), float("inf")):
        q2 = q.clone()
        q2[0, 77, 1] = bad
        o, lse = ut.xattn_fwd(q2, k, v, 0.1)
        dq = ut.xattn_bwd(q2, k, v, o, do, lse, 0.1)[0]
        others = torch.ones(200, 4, dtype=torch.bool, device=DEV)
        others[77, 1] = False
        assert torch.equal(o[0][others], want[0][0][others]) and torch.equal(dq[0][others], want[2][0][0][others])
        assert torch.equal(lse[0].T[others], want[1][0].T[others])


def test_masks_at_any_address_and_as_bool():
    q, k, v, do = draw(7, 1, 30, 1111, 2, 2, 64)
    m = make_mask("random", 1, 1111, 9)
    want = ut.xattn_fwd(q, k, v, 0.125, key_mask=torch.from_numpy(m).to(DEV))
    for shift in (1, 3, 7, 13):
        buf = torch.full((1111 + 16,), 1, dtype=torch.uint8, device=DEV)
        view = buf[shift:shift + 1111].view(1, 1111)
        view.copy_(torch.from_numpy(m))
        got = ut.xattn_fwd(q, k, v, 0.125, key_mask=view)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    got = ut.xattn_fwd(q, k, v, 0.125, key_mask=torch.from_numpy(m != 0).to(DEV))
    assert torch.equal(got[0], want[0])


def test_an_all_ones_mask_equals_no_mask():
    q, k, v, do = draw(8, 2, 100, 777, 4, 2, 128)
    a, b = run(q, k, v, do, 0.1, None), run(q, k, v, do, 0.1, np.ones((2, 777), np.uint8))
    for x, y in zip((a[0], a[1]) + a[2], (b[0], b[1]) + b[2]):
        assert torch.equal(x, y)


def test_strided_views_in_and_out():
    """Queries, keys, values and all outputs inside fused tensors; what lies
    between the rows stays."""
    B, Nq, Nk, Hq, Hk, D = 2, 90, 150, 4, 2, 64
    q, k, v, do = draw(9, B, Nq, Nk, Hq, Hk, D)
    o, lse, grads = run(q, k, v, do, 0.125, None)
    big = torch.full((B, Nq, 5, Hq, D), 3.0, dtype=torch.bfloat16, device=DEV)
    kv = torch.full((B, Nk, 5, Hk, D), 3.0, dtype=torch.bfloat16, device=DEV)
    big[:, :, 0], big[:, :, 2], kv[:, :, 0], kv[:, :, 1] = q, do, k, v
    l2 = torch.empty_like(lse)
    assert ut.ut_xattn_fwd(big[:, :, 0], kv[:, :, 0], kv[:, :, 1], big[:, :, 1], l2, 0.125) == ut.UT_OK
    ws = torch.empty(ut.ut_xattn_bwd_workspace_size(B, Nq, Nk, Hq, Hk, D), dtype=torch.uint8, device=DEV)
    assert ut.ut_xattn_bwd(big[:, :, 0], kv[:, :, 0], kv[:, :, 1], big[:, :, 1], big[:, :, 2], l2, big[:, :, 3],
                           kv[:, :, 2], kv[:, :, 3], 0.125, workspace=ws) == ut.UT_OK
    for x, y in ((big[:, :, 1], o), (l2, lse), (big[:, :, 3], grads[0]), (kv[:, :, 2], grads[1]), (kv[:, :, 3], grads[2])):
        assert torch.equal(x, y)
    assert (big[:, :, 4] == 3).all() and (kv[:, :, 4] == 3).all()
    assert torch.equal(big[:, :, 0], q) and torch.equal(kv[:, :, 1], v)


def test_keys_past_32_bit_offsets():
    """A cache whose rows lie 2^22 - 8 elements apart: keys 5 GB from the first."""
    Nk, stride, H, D = 600, (1 << 22) - 8, 1, 64
    g = torch.Generator(device=DEV).manual_seed(4)
    k, v = (torch.randn(1, Nk, H, D, generator=g, device=DEV).to(torch.bfloat16) for _ in range(2))
    q, do = (torch.randn(1, 50, H, D, generator=g, device=DEV).to(torch.bfloat16) for _ in range(2))
    buf = torch.empty((Nk - 1) * stride + 2 * D, dtype=torch.bfloat16, device=DEV)
    kf = torch.as_strided(buf, (1, Nk, H, D), (Nk * stride, stride, D, 1))
    vf = torch.as_strided(buf, (1, Nk, H, D), (Nk * stride, stride, D, 1), D)
    kf.copy_(k), vf.copy_(v)
    a, b = run(q, k, v, do, 0.125, None), run(q, kf, vf, do, 0.125, None)
    for x, y in zip((a[0], a[1]) + a[2], (b[0], b[1]) + b[2]):
        assert torch.equal(x, y)


def test_zero_lengths():
    q, k, v, do = draw(10, 2, 5, 0, 2, 1, 64)
    o, lse, (dq, dk, dv) = run(q, k, v, do, 0.125, None)
    assert (o == 0).all() and (lse == -math.inf).all() and (dq == 0).all() and dk.shape == k.shape
    q, k, v, do = draw(10, 2, 0, 70, 2, 1, 64)
    o, lse, (dq, dk, dv) = run(q, k, v, do, 0.125, None)
    assert o.numel() == 0 and dq.numel() == 0 and (dk == 0).all() and (dv == 0).all()


@pytest.mark.parametrize("Nk", [1, 2, 3, 33, 64])
@pytest.mark.parametrize("Hq,Hk,D", [(4, 2, 64), (3, 1, 128)])
def test_few_keys_do_not_feel_the_rounding_of_o(Nk, Hq, Hk, D):
    """dP - delta is a small difference there. Bounds by element: dS and the results
    are rounded to bf16 (u = 2^-8 each); P, dP and delta are fp32, off by less than
    2^-16 of the sums of magnitudes that they are formed from."""
    q, k, v, do = draw(12, 1, 300, Nk, Hq, Hk, D)
    scale = D ** -0.5
    _, _, (dq, dk, dv) = run(q, k, v, do, scale, None)
    Q, DO = (x[0].double().cpu().permute(1, 0, 2) for x in (q, do))                       # [Hq, Nq, D]
    K, V = (x[0].double().cpu().permute(1, 0, 2).repeat_interleave(Hq // Hk, 0) for x in (k, v))
    P = (Q @ K.mT * scale).softmax(-1)
    dP, adP = DO @ V.mT, DO.abs() @ V.abs().mT
    dS = P * (dP - (P * dP).sum(-1, keepdim=True))
    u = 2.0 ** -8
    eS = u * dS.abs() + 2.0 ** -16 * P * (adP + (P * adP).sum(-1, keepdim=True))
    shared = lambda x: x.unflatten(0, (Hk, -1)).sum(1)  # noqa: E731
    for name, got, ref, err in (("dq", dq, scale * (dS @ K), scale * (eS @ K.abs())),
                                ("dk", dk, shared(scale * (dS.mT @ Q)), shared(scale * (eS.mT @ Q.abs())))):
        got = got[0].double().cpu().permute(1, 0, 2)
        worst = ((got - ref).abs() / (u * ref.abs() + (1 + u) * err)).max().item()
        assert worst <= 1, (name, worst)


def test_query_rows_past_32_bit_offsets():
    """Rows of queries and results 2^22 - 8 elements apart, the last tile cut short."""
    for Nq, Hq, Hk in ((290, 1, 1), (258, 3, 1)):
        D, stride, width = 64, (1 << 22) - 8, 3 * 64
        q, k, v, do = draw(13, 1, Nq, 100, Hq, Hk, D)
        want = run(q, k, v, do, 0.125, None)
        buf = torch.zeros((Nq - 1) * stride + 4 * width, dtype=torch.bfloat16, device=DEV)
        at = lambda i: torch.as_strided(buf, (1, Nq, Hq, D), (Nq * stride, stride, D, 1), i * width)  # noqa: E731
        at(0).copy_(q), at(1).copy_(do)
        lse, dk, dv = torch.empty_like(want[1]), torch.empty_like(k), torch.empty_like(v)
        assert ut.ut_xattn_fwd(at(0), k, v, at(2), lse, 0.125) == ut.UT_OK
        ws = torch.empty(ut.ut_xattn_bwd_workspace_size(1, Nq, 100, Hq, Hk, D), dtype=torch.uint8, device=DEV)
        assert ut.ut_xattn_bwd(at(0), k, v, at(2), at(1), lse, at(3), dk, dv, 0.125, workspace=ws) == ut.UT_OK
        for x, y in ((at(2), want[0]), (lse, want[1]), (at(3), want[2][0]), (dk, want[2][1]), (dv, want[2][2])):
            assert torch.equal(x, y)
        assert torch.equal(at(0), q) and torch.equal(at(1), do)
        assert int(torch.count_nonzero(buf)) <= 4 * Nq * Hq * D   # nothing between the rows was written
        del buf, at


# ---- packed samples --------------------------------------------------------

def offsets(lens):
    return torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device=DEV)


def packed(seed, lq, lk, Hq, Hk, D, rest=0, kind=None):
    g = torch.Generator().manual_seed(seed)
    r = lambda n, h: torch.randn((n, h, D), generator=g).to(torch.bfloat16).to(DEV)  # noqa: E731
    Tq, Tk = sum(lq) + rest, sum(lk) + rest
    q, do, k, v = r(Tq, Hq), r(Tq, Hq), r(Tk, Hk), r(Tk, Hk)
    mask = None if kind is None else make_mask(kind, 1, Tk, seed)[0]
    return q, k, v, do, mask


VARLEN = [  # lq, lk, Hq, Hk, D
    ([70, 130, 1, 33], [20, 64, 65, 1], 4, 2, 64), ([5, 0, 300], [0, 77, 129], 2, 2, 128), ([1] * 6, [700] * 6, 8, 2, 128),
    ([200], [300], 3, 1, 72), ([0, 0, 40], [50, 0, 9], 2, 1, 40), ([1, 2, 3], [4200, 1, 9000], 4, 1, 64),
    ([900, 800], [10, 17], 2, 2, 128),
]


@pytest.mark.parametrize("kind", [None, "random"])
@pytest.mark.parametrize("lq,lk,Hq,Hk,D", VARLEN)
def test_varlen_matches_oracle(lq, lk, Hq, Hk, D, kind):
    rest = 13
    q, k, v, do, mask = packed(20, lq, lk, Hq, Hk, D, rest, kind)
    m = None if mask is None else torch.from_numpy(mask).to(DEV)
    scale = 1 / math.sqrt(D)
    at = (offsets(lq), max(lq), offsets(lk), max(lk))
    o, lse = ut.xattn_fwd_varlen(q, k, v, *at, scale, key_mask=m)
    grads = ut.xattn_bwd_varlen(q, k, v, o, do, lse, *at, scale, key_mask=m)
    torch.cuda.synchronize()
    eq, ek = np.concatenate([[0], np.cumsum(lq)]), np.concatenate([[0], np.cumsum(lk)])
    for b in range(len(lq)):
        sq, sk = slice(eq[b], eq[b + 1]), slice(ek[b], ek[b + 1])
        check(*(f64(x[s])[None] for x, s in ((q, sq), (k, sk), (v, sk), (do, sq))), scale,
              None if mask is None else mask[sk][None], f64(o[sq])[None], f64(lse[:, sq])[None],
              [f64(grads[0][sq])[None], f64(grads[1][sk])[None], f64(grads[2][sk])[None]], f"sample {b}")
    # rows behind the last sample
    assert (o[eq[-1]:] == 0).all() and (lse[:, eq[-1]:] == -math.inf).all() and (grads[0][eq[-1]:] == 0).all()
    assert (grads[1][ek[-1]:] == 0).all() and (grads[2][ek[-1]:] == 0).all()


@pytest.mark.parametrize("lq,lk", [([70, 9], [40, 300]), ([1, 1], [4500, 4500]), ([1500], [20])])
def test_varlen_rows_of_no_sample_stay_as_they_were(lq, lk):
    q, k, v, do, _ = packed(21, lq, lk, 2, 1, 64, 29)
    o, dq, dk, dv = (torch.full_like(x, 5.0) for x in (q, q, k, v))
    lse = torch.full((2, q.shape[0]), 5.0, device=DEV)
    at = (offsets(lq), max(lq), offsets(lk), max(lk))
    wsf = torch.empty(max(16, ut.ut_xattn_fwd_varlen_workspace_size(len(lq), q.shape[0], max(lq), max(lk), 2, 1, 64)),
                      dtype=torch.uint8, device=DEV)
    wsb = torch.empty(ut.ut_xattn_bwd_varlen_workspace_size(len(lq), q.shape[0], k.shape[0], max(lq), max(lk), 2, 1, 64),
                      dtype=torch.uint8, device=DEV)
    assert ut.ut_xattn_fwd_varlen(q, k, v, o, lse, *at, 0.1, workspace=wsf) == ut.UT_OK
    assert ut.ut_xattn_bwd_varlen(q, k, v, o, do, lse, dq, dk, dv, *at, 0.1, workspace=wsb) == ut.UT_OK
    eq, ek = sum(lq), sum(lk)
    for x, e in ((o, eq), (dq, eq), (dk, ek), (dv, ek)):
        assert (x[e:] == 5).all() and not (x[:e] == 5).all()
    assert (lse[:, eq:] == 5).all()
    want = ut.xattn_fwd_varlen(q, k, v, *at, 0.1)
    assert torch.equal(want[0][:eq], o[:eq])


def test_varlen_of_equal_lengths_equals_the_uniform_call():
    B, Nq, Nk, Hq, Hk, D = 3, 130, 90, 4, 2, 128
    q, k, v, do = draw(22, B, Nq, Nk, Hq, Hk, D)
    a = run(q, k, v, do, 0.09, None)
    p = [x.reshape(-1, x.shape[2], D) for x in (q, k, v, do)]
    at = (offsets([Nq] * B), Nq, offsets([Nk] * B), Nk)
    o, lse = ut.xattn_fwd_varlen(p[0], p[1], p[2], *at, 0.09)
    grads = ut.xattn_bwd_varlen(p[0], p[1], p[2], o, p[3], lse, *at, 0.09)
    assert torch.equal(o.view(a[0].shape), a[0])
    assert torch.equal(lse.view(Hq, B, Nq).permute(1, 0, 2), a[1])
    for x, y in zip(grads, a[2]):
        assert torch.equal(x.view(y.shape), y)


@pytest.mark.parametrize("B,Hq,Hk,D", [(9000, 8, 8, 16), (2500, 8, 2, 128)])
def test_many_short_samples(B, Hq, Hk, D):
    """More items a workgroup than one group of its item numbers holds. Bounds by
    element: P, dS, O (which forms delta) and every result are off by half a step of
    bf16 each, u = 2^-8; fp32's own errors are below 2^-16 of the same sums."""
    g = torch.Generator().manual_seed(B)
    lq, lk = (torch.randint(0, n, (B,), generator=g) for n in (4, 5))
    eq, ek = ([0] + x.cumsum(0).tolist() for x in (lq, lk))
    q, do = (torch.randn(eq[-1], Hq, D, generator=g).bfloat16() for _ in range(2))
    k, v = (torch.randn(ek[-1], Hk, D, generator=g).bfloat16() for _ in range(2))
    at = (torch.tensor(eq, dtype=torch.int32, device=DEV), 3, torch.tensor(ek, dtype=torch.int32, device=DEV), 4)
    scale = D ** -0.5
    dev = [x.to(DEV) for x in (q, k, v, do)]
    o, lse = ut.xattn_fwd_varlen(*dev[:3], *at, scale)
    dq, dk, dv = ut.xattn_bwd_varlen(*dev[:3], o, dev[3], lse, *at, scale)

    def pad(x, ends, n):   # [B, H, n, D] in fp64, heads repeated to Hq
        out = torch.zeros(B, n, *x.shape[1:], dtype=torch.float64)
        for i in range(n):
            has = torch.tensor(ends[1:]) - torch.tensor(ends[:-1]) > i
            out[has, i] = x.double()[torch.tensor(ends[:-1])[has] + i]
        return out.permute(0, 2, 1, 3).repeat_interleave(Hq // x.shape[1], 1)

    def flat(x, ends, H):   # back to [T, H, D], shared heads summed
        x = x.unflatten(1, (H, -1)).sum(2).permute(0, 2, 1, 3)
        n = torch.tensor(ends[1:]) - torch.tensor(ends[:-1])
        return x[torch.arange(x.shape[1]) < n[:, None]]

    Q, K, V, DO = pad(q, eq, 3), pad(k, ek, 4), pad(v, ek, 4), pad(do, eq, 3)
    used = (torch.arange(4) < lk[:, None])[:, None, None] & (torch.arange(3) < lq[:, None])[:, None, :, None]
    S = (Q @ K.mT * scale).masked_fill(~used, -math.inf)
    top = S.amax(-1, keepdim=True).clamp_min(-1e300)
    E = (S - top).exp()
    L = E.sum(-1, keepdim=True)
    P = E / L.clamp_min(1e-300)
    u, f = 2.0 ** -8, 1 + 2.0 ** -8
    O, aO = P @ V, P @ V.abs()
    dP = DO @ V.mT
    dS = P * (dP - (DO * O).sum(-1, keepdim=True))
    # the error of dS: its own rounding, and delta's through O (twice rounded)
    eS = u * dS.abs() + P * (2 * u * f) * (DO.abs() * aO).sum(-1, keepdim=True)
    want = {"o": (o, flat(O, eq, Hq), flat(2 * u * f * aO, eq, Hq)),
            "dq": (dq, flat(scale * (dS @ K), eq, Hq), flat(scale * f * (eS @ K.abs()), eq, Hq)),
            "dk": (dk, flat(scale * (dS.mT @ Q), ek, Hk), flat(scale * f * (eS.mT @ Q.abs()), ek, Hk)),
            "dv": (dv, flat(P.mT @ DO, ek, Hk), flat(u * f * (P.mT @ DO.abs()), ek, Hk))}
    for name, (got, ref, bound) in want.items():
        got = got.cpu().double()
        bound = bound + u * ref.abs() + 2.0 ** -16 * (1 + bound / u)
        worst = ((got - ref).abs() / bound).max().item()
        assert worst <= 1, (name, worst)
    want_lse = (top + L.clamp_min(1e-300).log()).squeeze(-1).masked_fill(~used.any(-1), -math.inf)
    want_lse = want_lse.permute(0, 2, 1)[torch.arange(3) < lq[:, None]].T   # [Hq, T]
    got = lse.cpu().double()
    assert torch.equal(got == -math.inf, want_lse == -math.inf)
    live = got != -math.inf
    assert (got - want_lse)[live].abs().max() < 1e-4


@pytest.mark.parametrize("lq,lk", [([0, 0], [30, 4]), ([30, 9], [0, 0]), ([0], [0])])
def test_varlen_sides_without_tokens(lq, lk):
    """All rows of an empty side lie behind the last sample."""
    q, k, v, do, _ = packed(22, lq, lk, 4, 2, 64, rest=21)
    at = (offsets(lq), max(lq), offsets(lk), max(lk))
    for _ in range(2):   # old values in the memory that the allocator hands out
        junk = [torch.full_like(x, 3.0) for x in (q, q, k, v)]
        del junk
        o, lse = ut.xattn_fwd_varlen(q, k, v, *at, 0.125)
        dq, dk, dv = ut.xattn_bwd_varlen(q, k, v, o, do, lse, *at, 0.125)
        for x in (o, dq, dk, dv):
            assert (x == 0).all()
        assert (lse == -math.inf).all()


def test_bad_offsets_reach_nothing_outside():
    """Offsets outside the tensors are clamped (and refused in validate mode)."""
    q, k, v, do, _ = packed(23, [50, 50], [40, 40], 2, 2, 64)
    bad_q = torch.tensor([-7, 60, 5000], dtype=torch.int32, device=DEV)
    bad_k = torch.tensor([90, 20, 1 << 30], dtype=torch.int32, device=DEV)
    o, lse = ut.xattn_fwd_varlen(q, k, v, bad_q, 50, bad_k, 40, 0.1)
    ut.xattn_bwd_varlen(q, k, v, o, do, torch.zeros_like(lse), bad_q, 50, bad_k, 40, 0.1)
    torch.cuda.synchronize()


def test_validate_mode_checks_the_offsets(monkeypatch):
    q, k, v, do, _ = packed(24, [50, 50], [40, 40], 2, 2, 64, 5)
    good = (offsets([50, 50]), 50, offsets([40, 40]), 40)
    monkeypatch.setenv("UT_VALIDATE", "1")
    want = ut.xattn_fwd_varlen(q, k, v, *good, 0.1)
    for at in ((offsets([50, 500]), 50, good[2], 40), (good[0], 49, good[2], 40), (good[0], 50, offsets([40, -3]), 40),
               (good[0], 50, good[2] + 1, 40)):
        with pytest.raises(ut.UltraTexError) as e:
            ut.xattn_fwd_varlen(q, k, v, *at, 0.1)
        assert e.value.status == ut.UT_ERR_INVALID_ARG
    assert want[0].shape == q.shape


# ---- streams, graphs, repeated runs ----------------------------------------

@pytest.mark.parametrize("Nq,Nk", [(1, 5000), (600, 100)])
def test_equal_results_on_every_run_and_on_a_side_stream(Nq, Nk):
    q, k, v, do = draw(30, 2, Nq, Nk, 4, 2, 128)
    a = run(q, k, v, do, 0.1, None)
    side = torch.cuda.Stream()
    b = run(q, k, v, do, 0.1, None, stream=side)
    for x, y in zip((a[0], a[1]) + a[2], (b[0], b[1]) + b[2]):
        assert torch.equal(x, y)


def test_two_calls_at_once():
    """On two streams, each with workspaces of its own: what they write stays their own."""
    data = [draw(33 + i, 2, Nq, Nk, 4, 2, 64 + 64 * i) for i, (Nq, Nk) in enumerate([(3000, 130), (30, 4000)])]
    want = [run(*d, 0.1, None) for d in data]
    sides = [torch.cuda.Stream() for _ in data]
    got = [[], []]
    for _ in range(4):
        for i, (q, k, v, do) in enumerate(data):
            o, lse = ut.xattn_fwd(q, k, v, 0.1, stream=sides[i])
            got[i].append((o, lse) + tuple(ut.xattn_bwd(q, k, v, o, do, lse, 0.1, stream=sides[i])))
    torch.cuda.synchronize()
    for i in range(2):
        for g in got[i]:
            for x, y in zip(g, (want[i][0], want[i][1]) + tuple(want[i][2])):
                assert torch.equal(x, y)


@pytest.mark.parametrize("Nq,Nk", [(1, 5000), (600, 100), (77, 130)])
def test_captured_and_replayed(Nq, Nk):
    q, k, v, do = draw(31, 2, Nq, Nk, 4, 2, 64)
    m = torch.from_numpy(make_mask("random", 2, Nk, 3)).to(DEV)

    def both():
        o, lse = ut.xattn_fwd(q, k, v, 0.125, key_mask=m)
        return (o, lse) + ut.xattn_bwd(q, k, v, o, do, lse, 0.125, key_mask=m)

    both()
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    outs = []
    for graph in graphs:
        with torch.cuda.graph(graph):
            outs.append(both())
    for i in range(3):
        q.mul_(-0.75)
        m.copy_(m.roll(17, 1))
        for graph in graphs:
            graph.replay()
        want = both()
        torch.cuda.synchronize()
        for out in outs:
            for x, y in zip(out, want):
                assert torch.equal(x, y), i


def test_workspace_contents_do_not_matter():
    for Nq, Nk in ((1, 5000), (2000, 40)):
        q, k, v, do = draw(32, 1, Nq, Nk, 2, 2, 64)
        want = run(q, k, v, do, 0.125, None)
        wf = torch.full((max(16, ut.ut_xattn_fwd_workspace_size(1, Nq, Nk, 2, 2, 64)),), 255, dtype=torch.uint8, device=DEV)
        wb = torch.full((ut.ut_xattn_bwd_workspace_size(1, Nq, Nk, 2, 2, 64),), 255, dtype=torch.uint8, device=DEV)
        o, lse = ut.xattn_fwd(q, k, v, 0.125, workspace=wf)
        grads = ut.xattn_bwd(q, k, v, o, do, lse, 0.125, workspace=wb)
        assert torch.equal(o, want[0]) and torch.equal(lse, want[1])
        for x, y in zip(grads, want[2]):
            assert torch.equal(x, y)


def test_full_size_rows_of_the_2k_layer():
    """The 2048-canvas layer against 512 text tokens, one head checked: forward
    and dQ rows at both ends, dK and dV from all 77,060 rows."""
    Nq, Nk, H, D = 77060, 512, 24, 128
    g = torch.Generator(device=DEV).manual_seed(5)
    q, do = (torch.randn(1, Nq, H, D, generator=g, device=DEV).to(torch.bfloat16) for _ in range(2))
    kv = torch.randn(1, Nk, 2, H, D, generator=g, device=DEV).to(torch.bfloat16)
    scale = 1 / math.sqrt(D)
    o, lse, (dq, dk, dv) = run(q, kv[:, :, 0], kv[:, :, 1], do, scale, None)
    h = 17
    Q, K, V, G = (x[0, :, h].double() for x in (q, kv[:, :, 0], kv[:, :, 1], do))
    S = Q @ K.T * scale
    L = torch.logsumexp(S, 1)
    P = torch.exp(S - L[:, None])
    O = P @ V
    dS = P * (G @ V.T - (G * O).sum(1, keepdim=True))
    assert (lse[0, h].double() - L).abs().max() <= 1e-3
    for got, ref, lim in ((o, O, 1e-2), (dq, dS @ K * scale, 2e-2), (dk, dS.T @ Q * scale, 2e-2), (dv, P.T @ G, 2e-2)):
        x = got[0, :, h].double()
        assert (x - ref).norm() <= lim * ref.norm()
        assert (x - ref).abs().max() <= 2e-2 * ref.abs().max()


def test_views_broadcast_over_tokens_or_samples_are_refused():
    """Refused on the host, inputs and outputs alike; a copy of such a view is fine."""
    q, k, v, do = draw(40, 2, 30, 20, 4, 2, 64)
    o, lse = ut.xattn_fwd(q, k, v, 0.125)
    flat = [x[0] for x in (q, k, v, do)]
    at = (offsets([30]), 30, offsets([20]), 20)
    one_q, one_k, one_do = q[:1, :1].expand(2, 1, 4, 64), k[:1, :1].expand(1, 20, 2, 64), do[:1, :1].expand(1, 30, 4, 64)
    pos = torch.zeros(30, 1, device=DEV)
    for call in (lambda: ut.xattn_fwd(one_q, k, v, 0.125),
                 lambda: ut.xattn_fwd(q[:1], one_k, one_k, 0.125),
                 lambda: ut.xattn_bwd(q[:1], k[:1], v[:1], o[:1], one_do, lse[:1], 0.125),
                 lambda: ut.xattn_fwd_varlen(flat[0], one_k[0], flat[2], *at, 0.125),
                 lambda: ut.xattn_bwd_varlen(*flat[:3], o[0], one_do[0], lse[0], *at, 0.125),
                 lambda: ut.ut_xattn_fwd(q[:1], k[:1], v[:1], one_do, lse[:1], 0.125),
                 lambda: ut.qk_rope_fwd(one_do, None, pos, (64,)),
                 lambda: ut.qk_rope_bwd(q[0], one_do[0], pos, (64,))):
        with pytest.raises(ValueError, match="tokens overlap"):
            call()
    want = ut.xattn_bwd(q[:1], k[:1], v[:1], o[:1], one_do.contiguous(), lse[:1], 0.125)
    check_do = do[:1, :1].repeat(1, 30, 1, 1)
    for x, y in zip(want, ut.xattn_bwd(q[:1], k[:1], v[:1], o[:1], check_do, lse[:1], 0.125)):
        assert torch.equal(x, y)


@pytest.mark.parametrize("zero_rest", [False, True])
@pytest.mark.parametrize("bad_q,bad_k", [([-7, 60, 5000], [90, 20, 1 << 30]), ([0, 100, 40], [0, 80, -5]),
                                         ([99, 99, 101], [79, 1000, 80]), ([-(1 << 31), 0, (1 << 31) - 1],) * 2])
@pytest.mark.parametrize("maxq,maxk,Hq,Hk,D", [(50, 40, 2, 2, 64), (50, 4000, 4, 2, 128), (4000, 40, 2, 1, 72)])
def test_bad_offsets_write_nothing_outside(bad_q, bad_k, maxq, maxk, Hq, Hk, D, zero_rest):
    """Every buffer that the calls write lies between margins, which stay as they were (the longer
    maxima split the keys or the query rows, so that the workspaces hold partial results)."""
    q, k, v, do, _ = packed(41, [50, 50], [40, 40], Hq, Hk, D)
    cq, ck = (torch.tensor(x, dtype=torch.int32, device=DEV) for x in (bad_q, bad_k))
    margin, held = 1 << 14, []

    def inside(shape, dtype):
        n = math.prod(shape)
        buf = torch.full((n + 2 * margin,), 77, dtype=dtype, device=DEV)
        held.append((buf, n))
        return buf[margin:margin + n].view(shape)

    o, dq, dk, dv = (inside(x.shape, torch.bfloat16) for x in (q, q, k, v))
    lse = inside((Hq, 100), torch.float32)
    wf = inside((max(16, ut.ut_xattn_fwd_varlen_workspace_size(2, 100, maxq, maxk, Hq, Hk, D)),), torch.uint8)
    wb = inside((ut.ut_xattn_bwd_varlen_workspace_size(2, 100, 80, maxq, maxk, Hq, Hk, D),), torch.uint8)
    ins = [x.clone() for x in (q, k, v, do)]
    at = (cq, maxq, ck, maxk, 0.1)
    assert ut.ut_xattn_fwd_varlen(q, k, v, o, lse, *at, zero_rest=zero_rest, workspace=wf) == ut.UT_OK
    assert ut.ut_xattn_bwd_varlen(q, k, v, o, do, lse, dq, dk, dv, *at, zero_rest=zero_rest, workspace=wb) == ut.UT_OK
    torch.cuda.synchronize()
    for buf, n in held:
        assert (buf[:margin] == 77).all() and (buf[margin + n:] == 77).all()
    for x, y in zip((q, k, v, do), ins):
        assert torch.equal(x, y)


def few_keys_bounds(q, k, v, do, used, scale, dq, dk, label):
    """Gradients of one sample [N, H, D] whose keys `used` are in use, with the bounds of
    test_few_keys_do_not_feel_the_rounding_of_o: delta has no share of a rounded O."""
    Hq, Hk = q.shape[1], k.shape[1]
    Q, DO = (x.double().cpu().permute(1, 0, 2) for x in (q, do))
    K, V = (x[used].double().cpu().permute(1, 0, 2).repeat_interleave(Hq // Hk, 0) for x in (k, v))
    P = (Q @ K.mT * scale).softmax(-1)
    dP, adP = DO @ V.mT, DO.abs() @ V.abs().mT
    dS = P * (dP - (P * dP).sum(-1, keepdim=True))
    u = 2.0 ** -8
    eS = u * dS.abs() + 2.0 ** -16 * P * (adP + (P * adP).sum(-1, keepdim=True))
    shared = lambda x: x.unflatten(0, (Hk, -1)).sum(1)  # noqa: E731
    for name, got, ref, err in (("dq", dq, scale * (dS @ K), scale * (eS @ K.abs())),
                                ("dk", dk[used], shared(scale * (dS.mT @ Q)), shared(scale * (eS.mT @ Q.abs())))):
        got = got.double().cpu().permute(1, 0, 2)
        worst = ((got - ref).abs() / (u * ref.abs() + (1 + u) * err)).max().item()
        assert worst <= 1, (label, name, worst)


# (keys in use, from where) of each sample: within one 64-key tile each time; a key
# of its own at both ends. Rows and keys: unsplit and split work, more than 64 tiles
# of 64 keys (a lane each), a sample whose tile lies behind them.
@pytest.mark.parametrize("used", [[(1, 0), (2, 130)], [(33, 64), (64, 192)], [(1, -1), (7, 249)]])
@pytest.mark.parametrize("Nq,Nk,Hq,Hk,D", [(300, 300, 4, 2, 64), (300, 300, 3, 1, 128), (300, 1030, 4, 2, 64),
                                           (5, 9001, 4, 2, 128), (2100, 4500, 32, 16, 64)])
def test_few_keys_in_use_do_not_feel_the_rounding_of_o(Nq, Nk, Hq, Hk, D, used):
    q, k, v, do = draw(42, 2, Nq, Nk, Hq, Hk, D)
    mask = np.zeros((2, Nk), np.uint8)
    for b, (n, at) in enumerate(used):
        at = at if at >= 0 else Nk + at
        mask[b, at:at + n] = 1
    scale = D ** -0.5
    _, _, (dq, dk, _) = run(q, k, v, do, scale, mask)
    for b in range(2):
        few_keys_bounds(q[b], k[b], v[b], do[b], np.flatnonzero(mask[b]), scale, dq[b], dk[b], (b, used[b]))


def test_few_keys_of_packed_and_padded_prompts_give_equal_gradients():
    """The same prompts packed (21 and 64 keys) and padded to 300: one arithmetic."""
    lk, Nq, Nk, Hq, Hk, D = [21, 64], 150, 300, 4, 2, 64
    q, k, v, do = draw(43, 2, Nq, Nk, Hq, Hk, D)
    mask = np.zeros((2, Nk), np.uint8)
    for b, n in enumerate(lk):
        mask[b, :n] = 1
    _, _, (dq, dk, dv) = run(q, k, v, do, 0.125, mask)
    at = (offsets([Nq] * 2), Nq, offsets(lk), max(lk))
    kp, vp = (torch.cat([x[b, :n] for b, n in enumerate(lk)]) for x in (k, v))
    o, lse = ut.xattn_fwd_varlen(q.flatten(0, 1), kp, vp, *at, 0.125)
    want = ut.xattn_bwd_varlen(q.flatten(0, 1), kp, vp, o, do.flatten(0, 1), lse, *at, 0.125)
    assert torch.equal(dq.flatten(0, 1), want[0])
    for x, y in ((dk, want[1]), (dv, want[2])):
        assert torch.equal(torch.cat([x[b, :n] for b, n in enumerate(lk)]), y)


@pytest.mark.parametrize("Nq,Nk", [(40, 700), (300, 300), (5, 9001)])
def test_few_keys_of_samples_with_and_without_any(Nq, Nk):
    """Of five samples one has no key in use, two have keys in one tile, two in two tiles; the
    statistics of the dQ pass serve the dK and dV of each."""
    q, k, v, do = draw(44, 5, Nq, Nk, 4, 2, 64)
    mask = np.zeros((5, Nk), np.uint8)
    mask[1, 70:90] = 1
    mask[2, -3:] = 1
    mask[3, [0, Nk - 1]] = 1
    mask[4, 60:70] = 1
    o, lse, grads = run(q, k, v, do, 0.125, mask)
    check(*(f64(t) for t in (q, k, v, do)), 0.125, mask, f64(o), f64(lse), [f64(t) for t in grads], f"{(Nq, Nk)}")
    for b in (1, 2):
        few_keys_bounds(q[b], k[b], v[b], do[b], np.flatnonzero(mask[b]), 0.125, grads[0][b], grads[1][b], b)


def test_as_many_samples_as_a_launch_takes():
    """2^24 - 8 samples of one query and one key: O is V, dV is dO, and dQ and dK are 0 but
    for fp32's rounding."""
    B = (1 << 24) - 8
    g = torch.Generator(device=DEV).manual_seed(45)
    q, k, v, do = (torch.randn(B, 1, 1, 8, generator=g, device=DEV, dtype=torch.bfloat16) for _ in range(4))
    o, lse, (dq, dk, dv) = run(q, k, v, do, 0.25, None)
    assert torch.equal(o, v) and torch.equal(dv, do)
    # P = exp2(s - lse) is off by at most 2^-20 of 1, and dS = P dP - P rowsum(P dP) by that of |dP|
    dp = (do.float().abs() * v.float().abs()).sum(-1, keepdim=True)
    for got, x in ((dq, k), (dk, q)):
        assert (got.float().abs() <= 2.0 ** -18 * 0.25 * dp * x.float().abs()).all()
    want = (q.double() * k.double()).sum(-1)[:, 0] * 0.25
    assert (lse[:, 0, 0].double() - want[:, 0]).abs().max() <= 2.0 ** -16
    with pytest.raises(ut.UltraTexError) as e:
        ut.xattn_bwd(*(torch.cat([x, x[:1]]) for x in (q, k, v, o, do)), torch.zeros(B + 1, 1, 1, device=DEV), 0.25)
    assert e.value.status == ut.UT_ERR_INVALID_ARG
