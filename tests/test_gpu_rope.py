"""Rotary positions with the per-head norm on the GPU against the float64 oracle.

Tolerances, per element, u_t the half step of the stored type (bf16 2^-8, fp32
2^-24 relative):
  angle  the reduced angle is rounded to fp32 once, 2^-25 turns = 1.9e-7 rad, and
         cos and sin are within 2 ulp of 1: together below 4e-7;
  norm   a sum of D squares in fp32, a division, a square root and two products:
         (D/2 + 8) 2^-24 relative;
  out    |err| <= u_t |ref| + (|a| + |b|) ((D/2 + 12) 2^-24 + 4e-7), (a, b) the
         pair before the rotation;
  dx     rstd (g w - h mean(g w h)): the mean adds D products, so
         |err| <= u_t |ref| + rstd (|g w| + |h| mean|g w h|) ((2 D + 24) 2^-24 + 8e-7),
         |g| taken as the sum of the pair's two gradients;
  dw     N = tokens x heads products added in fp32 in some order:
         |err| <= sum|g h| ((N + D + 32) 2^-24 + 8e-7).
"""
import math

import numpy as np
import pytest
import torch

import oracle
import paper_2609_23169_amd as ut

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
E24 = 2.0 ** -24


def f64(t):
    return t.detach().double().cpu().numpy()


def pair_abs(x, R, interleaved):
    """|u| + |v| of each element's pair (|x| behind R)."""
    y = np.abs(x).copy()
    if interleaved:
        s = np.repeat(y[..., 0:R:2] + y[..., 1:R:2], 2, axis=-1)
    else:
        h = y[..., :R // 2] + y[..., R // 2:R]
        s = np.concatenate([h, h], -1)
    y[..., :R] = s
    return y


def case(seed, n, Hq, Hk, D, axes, dtype, kept=False, norm=True, rows=None, wdtype=None, fused=False):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g)  # noqa: E731
    if fused:
        proj = r(n, Hq + 2 * max(Hk, 1), D).to(dtype).to(DEV)
        q, k = proj[:, :Hq], proj[:, Hq:Hq + Hk]
    else:
        q, k = r(n, Hq, D).to(dtype).to(DEV), r(n, Hk, D).to(dtype).to(DEV)
    rows = rows or max(n, 1)
    pos = torch.randint(0, 200, (rows, len(axes)), generator=g).float() * 0.5
    c = {"q": q, "k": k if Hk else None, "dq": r(n, Hq, D).to(dtype).to(DEV),
         "dk": r(n, Hk, D).to(dtype).to(DEV) if Hk else None, "pos": pos.to(DEV), "axes": axes, "idx": None, "wq": None,
         "wk": None}
    if kept:
        c["idx"] = torch.randint(-2, rows + 2, (n,), generator=g, dtype=torch.int32).to(DEV)   # some outside
    if norm:
        c["wq"], c["wk"] = (1 + 0.3 * r(D)).to(wdtype or dtype).to(DEV), (1 + 0.3 * r(D)).to(wdtype or dtype).to(DEV)
        if not Hk:
            c["wk"] = None
    return c


def check(c, interleaved, theta=10000.0, eps=1e-6):
    kw = dict(theta=theta, token_idx=c["idx"], q_weight=c["wq"], k_weight=c["wk"], eps=eps, interleaved=interleaved)
    qo, ko = ut.qk_rope_fwd(c["q"], c["k"], c["pos"], c["axes"], **kw)
    dq, dk, dwq, dwk = ut.qk_rope_bwd(c["dq"], c["dk"], c["pos"], c["axes"], q=c["q"], k=c["k"], **kw)
    torch.cuda.synchronize()
    pos, idx, R = f64(c["pos"]), None if c["idx"] is None else c["idx"].cpu().numpy(), sum(c["axes"])
    for x, w, y, dy, dx, dw in ((c["q"], c["wq"], qo, c["dq"], dq, dwq), (c["k"], c["wk"], ko, c["dk"], dk, dwk)):
        if x is None:
            assert y is None and dx is None and dw is None
            continue
        D, u = x.shape[-1], U[x.dtype]
        X, G = f64(x), f64(dy)
        w64 = None if w is None else f64(w)
        ref = oracle.rope_fwd(X, pos, c["axes"], theta, idx, w64, eps, interleaved)
        rstd = 1 / np.sqrt((X * X).mean(-1, keepdims=True) + eps)
        hat = X if w is None else X * rstd * w64
        tol = u * np.abs(ref) + pair_abs(hat, R, interleaved) * ((D / 2 + 12) * E24 + 4e-7)
        assert y.dtype == x.dtype and y.is_contiguous()
        assert np.all(np.abs(f64(y) - ref) <= tol), float((np.abs(f64(y) - ref) / tol).max())
        rdx, rdw = oracle.rope_bwd(G, pos, c["axes"], theta, idx, X, w64, eps, interleaved)
        ga = pair_abs(G, R, interleaved)
        if w is None:
            tol = u * np.abs(rdx) + ga * ((D / 2 + 12) * E24 + 4e-7)
            assert dw is None
        else:
            h, gw = np.abs(X * rstd), ga * np.abs(w64)
            tol = u * np.abs(rdx) + rstd * (gw + h * (gw * h).mean(-1, keepdims=True)) * ((2 * D + 24) * E24 + 8e-7)
            N = X.shape[0] * X.shape[1]
            tw = (ga * h).sum((0, 1)) * ((N + D + 32) * E24 + 8e-7)
            assert dw.dtype == torch.float32
            assert np.all(np.abs(f64(dw) - rdw) <= tw), float((np.abs(f64(dw) - rdw) / tw).max())
        assert np.all(np.abs(f64(dx) - rdx) <= tol), float((np.abs(f64(dx) - rdx) / tol).max())


SHAPES = [  # n, Hq, Hk, D, axes
    (1, 1, 1, 8, (2,)), (1, 24, 24, 128, (16, 56, 56)), (2, 3, 0, 16, (4, 4, 4)), (77, 8, 2, 64, (16, 24, 24)),
    (130, 5, 5, 72, (24, 24, 24)), (63, 7, 1, 96, (32, 32)), (257, 4, 2, 128, (64, 64)), (33, 2, 2, 256, (64, 96, 96)),
    (19, 33, 3, 40, (8, 8, 8, 8)), (1500, 6, 3, 128, (16, 56, 56)), (5000, 2, 1, 32, (8, 12, 12)),
    (9, 300, 17, 24, (8,)), (40, 3, 2, 200, (40, 80, 80)),
]


@pytest.mark.parametrize("interleaved", [True, False])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n,Hq,Hk,D,axes", SHAPES)
def test_rope_matches_oracle(n, Hq, Hk, D, axes, dtype, interleaved):
    if not interleaved and sum(axes) % 8:
        axes = (8,) if D >= 8 else axes
    check(case(1, n, Hq, Hk, D, axes, dtype, kept=n % 2 == 1, norm=True), interleaved)
    check(case(2, n, Hq, Hk, D, axes, dtype, kept=n % 2 == 0, norm=False, rows=max(1, n // 3)), interleaved)


@pytest.mark.parametrize("axes", [(2, 4), (6, 10, 2), (62,)])
def test_near_pairs_that_end_inside_a_chunk(axes):
    check(case(3, 21, 3, 1, 64, axes, torch.float32), True)


def test_weights_of_another_dtype_and_fused_projection():
    check(case(4, 301, 6, 2, 128, (16, 56, 56), torch.bfloat16, wdtype=torch.float32, fused=True, kept=True), True)
    check(case(5, 44, 3, 3, 64, (16, 24, 24), torch.float32, wdtype=torch.bfloat16, fused=True), False)


def test_far_positions_keep_their_angles():
    """Positions of a million and more: the angle is formed in 64 bits."""
    c = case(6, 50, 2, 2, 64, (32, 32), torch.float32, norm=False)
    c["pos"] = (c["pos"] * 64 + 4_000_000).contiguous()
    check(c, True)


def test_scale_extremes_of_the_norm():
    c = case(7, 12, 2, 2, 64, (16, 24, 24), torch.float32)
    c["q"] *= torch.logspace(-12, 12, 12, device=DEV)[:, None, None]
    c["k"][3] = 0
    kw = dict(theta=10000.0, q_weight=c["wq"], k_weight=c["wk"], eps=1e-6)
    qo, ko = ut.qk_rope_fwd(c["q"], c["k"], c["pos"], c["axes"], **kw)
    assert torch.isfinite(qo).all() and torch.equal(ko[3], torch.zeros_like(ko[3]))
    ref = oracle.rope_fwd(f64(c["q"]), f64(c["pos"]), c["axes"], 10000.0, None, f64(c["wq"]), 1e-6)
    assert np.abs(f64(qo) - ref).max() <= 2e-5 * np.abs(ref).max()


def test_a_bad_row_stays_its_own():
    c = case(8, 40, 3, 1, 128, (16, 56, 56), torch.bfloat16)
    a = ut.qk_rope_fwd(c["q"], c["k"], c["pos"], c["axes"], q_weight=c["wq"], k_weight=c["wk"])
    c["q"][5, 1] = float("nan")
    c["pos"][7] = float("inf")
    b = ut.qk_rope_fwd(c["q"], c["k"], c["pos"], c["axes"], q_weight=c["wq"], k_weight=c["wk"])
    keep = torch.ones(40, 3, dtype=torch.bool, device=DEV)
    keep[5, 1] = False
    keep[7] = False
    assert torch.equal(a[0][keep], b[0][keep]) and torch.isnan(b[0][5, 1].float()).all()
    assert torch.isnan(b[0][7].float()).any()


@pytest.mark.parametrize("interleaved", [True, False])
@pytest.mark.parametrize("norm", [True, False])
def test_in_place_equals_out_of_place(norm, interleaved):
    c = case(9, 700, 5, 2, 64, (16, 24, 24), torch.bfloat16, kept=True, norm=norm, fused=True)
    kw = dict(theta=500.0, token_idx=c["idx"], q_weight=c["wq"], k_weight=c["wk"], interleaved=interleaved)
    want = ut.qk_rope_fwd(c["q"], c["k"], c["pos"], c["axes"], **kw)
    grads = ut.qk_rope_bwd(c["dq"], c["dk"], c["pos"], c["axes"], q=c["q"], k=c["k"], **kw)
    x, y = c["q"].clone(), c["k"].clone()
    dq, dk = c["dq"].clone(), c["dk"].clone()
    dwq, dwk = (torch.empty(64, device=DEV) for _ in range(2))
    ws = torch.empty(ut.ut_qk_rope_bwd_workspace_size(64), dtype=torch.uint8, device=DEV)
    assert ut.ut_qk_rope_bwd(dq, dk, x, y, dq, dk, c["pos"], c["axes"], dq_weight=dwq, dk_weight=dwk, workspace=ws,
                             **kw) == ut.UT_OK
    assert torch.equal(dq, grads[0]) and torch.equal(dk, grads[1])
    if norm:
        assert torch.equal(dwq, grads[2]) and torch.equal(dwk, grads[3])
    proj = torch.full((700, 9, 64), 7.0, dtype=torch.bfloat16, device=DEV)   # values behind stay
    proj[:, :5], proj[:, 5:7] = c["q"], c["k"]
    assert ut.ut_qk_rope_fwd(proj[:, :5], proj[:, 5:7], proj[:, :5], proj[:, 5:7], c["pos"], c["axes"], **kw) == ut.UT_OK
    assert torch.equal(proj[:, :5], want[0]) and torch.equal(proj[:, 5:7], want[1]) and (proj[:, 7:] == 7).all()


def test_batches_share_one_table_and_leading_dimensions():
    c = case(10, 60, 3, 1, 64, (16, 24, 24), torch.bfloat16, rows=20)
    kw = dict(q_weight=c["wq"], k_weight=c["wk"])
    a = ut.qk_rope_fwd(c["q"], c["k"], c["pos"], c["axes"], **kw)
    b = ut.qk_rope_fwd(c["q"].view(3, 20, 3, 64), c["k"].view(3, 20, 1, 64), c["pos"], c["axes"], **kw)
    assert b[0].shape == (3, 20, 3, 64)
    assert torch.equal(a[0], b[0].view(60, 3, 64)) and torch.equal(a[1], b[1].view(60, 1, 64))


def test_no_tokens():
    c = case(11, 0, 2, 2, 64, (16, 24, 24), torch.bfloat16)
    kw = dict(q_weight=c["wq"], k_weight=c["wk"])
    c["pos"] = torch.zeros(1, 3, device=DEV)
    assert ut.qk_rope_fwd(c["q"], c["k"], c["pos"], c["axes"], **kw)[0].shape == (0, 2, 64)
    out = ut.qk_rope_bwd(c["dq"], c["dk"], c["pos"], c["axes"], q=c["q"], k=c["k"], **kw)
    assert (out[2] == 0).all() and (out[3] == 0).all()


def test_rows_past_32_bit_offsets():
    """Tokens 2^30 elements and more from the first: 64-bit offsets in and out."""
    n, stride = 5, 1 << 30
    buf = torch.empty((n - 1) * stride + 128, dtype=torch.bfloat16, device=DEV)
    q = torch.as_strided(buf, (n, 2, 64), (stride, 64, 1))
    g = torch.Generator(device=DEV).manual_seed(3)
    q.copy_(torch.randn(n, 2, 64, generator=g, device=DEV))
    pos = torch.arange(n, device=DEV).float()[:, None].contiguous()
    want, _ = ut.qk_rope_fwd(q.contiguous(), None, pos, (64,))
    assert ut.ut_qk_rope_fwd(q, None, q, None, pos, (64,), 10000.0) == ut.UT_OK
    assert torch.equal(q.contiguous(), want)


def test_equal_results_on_every_run_and_on_a_side_stream():
    c = case(12, 9000, 4, 2, 128, (16, 56, 56), torch.bfloat16, kept=True)
    kw = dict(token_idx=c["idx"], q_weight=c["wq"], k_weight=c["wk"], q=c["q"], k=c["k"])
    a = ut.qk_rope_bwd(c["dq"], c["dk"], c["pos"], c["axes"], **kw)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    b = ut.qk_rope_bwd(c["dq"], c["dk"], c["pos"], c["axes"], stream=side, **kw)
    side.synchronize()
    for x, y in zip(a, b):
        assert torch.equal(x, y)


def test_captured_and_replayed():
    c = case(13, 500, 4, 2, 64, (16, 24, 24), torch.bfloat16, kept=True)
    kw = dict(token_idx=c["idx"], q_weight=c["wq"], k_weight=c["wk"])
    run = lambda: ut.qk_rope_fwd(c["q"], c["k"], c["pos"], c["axes"], **kw) + ut.qk_rope_bwd(  # noqa: E731
        c["dq"], c["dk"], c["pos"], c["axes"], q=c["q"], k=c["k"], **kw)
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = run()
    for i in range(3):
        c["q"].mul_(-0.5)
        c["dk"].add_(0.25)
        graph.replay()
        want = run()
        torch.cuda.synchronize()
        for x, y in zip(outs, want):
            assert torch.equal(x, y), i


def test_gradient_agrees_with_differences_of_the_forward():
    """Along random directions, the library's gradient against central
    differences of the oracle's forward: inside the gradient's own error."""
    c = case(14, 20, 2, 1, 64, (16, 24, 24), torch.float32)
    kw = dict(q_weight=c["wq"], k_weight=c["wk"])
    dq, _, dwq, _ = ut.qk_rope_bwd(c["dq"], c["dk"], c["pos"], c["axes"], q=c["q"], k=c["k"], **kw)
    X, G, w, pos = f64(c["q"]), f64(c["dq"]), f64(c["wq"]), f64(c["pos"])
    f = lambda x, y: float((oracle.rope_fwd(x, pos, c["axes"], 10000.0, None, y, 1e-6) * G).sum())  # noqa: E731
    rng = np.random.default_rng(1)
    for _ in range(3):
        ex, ew, h = rng.standard_normal(X.shape), rng.standard_normal(w.shape), 1e-4
        diff = (f(X + h * ex, w + h * ew) - f(X - h * ex, w - h * ew)) / (2 * h)
        got = float((f64(dq) * ex).sum() + (f64(dwq) * ew).sum())
        # h^2 of the difference and 2^-19 (about 160 roundings) of the gradient's terms
        size = float(np.abs(f64(dq) * ex).sum() + np.abs(f64(dwq) * ew).sum())
        assert abs(got - diff) <= size * (2.0 ** -19 + 1e-6), (got, diff, size)
    assert math.isfinite(got)
