"""How attention over a cache shares its work out, at the sizes where that changes:
four key heads at a time, more samples than a wave has lanes or the chip has
workgroups, parts of one row by the hundred, tiles of many rows with and without
parts; and calls that run at the same time. Against the float64 oracle, with the
tolerances of the cache's other tests."""
import pytest
import torch

import paper_2609_23169_amd as ut
from test_gpu_cache import check_attn, dev, rnd, words
from test_gpu_swattn import draw, offsets, run

pytestmark = pytest.mark.gpu
DEV = "cuda"


def ramp(B, most, seed):
    g = torch.Generator().manual_seed(seed)
    lens = torch.randint(0, most + 1, (B,), generator=g).tolist()
    lens[0], lens[-1] = most, 0
    return lens


def check(B, T, cap, lens, Hq, Hk, D, left, sinks, weighted=True, tree=None):
    q, k, v = rnd(60, B, T, Hq, D), rnd(61, B, cap, Hk, D), rnd(62, B, cap, Hk, D)
    w = torch.rand((B, Hk, cap), device=DEV) if weighted else None
    t = None if tree is None else torch.from_numpy(tree.view("int64")).to(DEV)
    got = ut.cache_attn(q, k, v, dev(lens), D ** -0.5, tree=t, window_left=left, n_sink=sinks, weights=w)
    check_attn(q, k, v, lens, D ** -0.5, got[0], got[1], tree, left, sinks, w, got[2] if weighted else None)


@pytest.mark.parametrize("weighted", [False, True])
@pytest.mark.parametrize("B,T,cap,lens,Hq,Hk,D,left,sinks", [
    (2, 1, 3100, [3099, 2500], 64, 64, 64, None, 0),    # a row a head
    (2, 1, 6200, [6199, 0], 64, 64, 64, 3500, 70),      # windows; an empty cache beside a long one
    (3, 2, 9000, [8998, 300, 7777], 60, 20, 128, None, 0),   # six rows, heads by five groups of four
    (2, 4, 13000, [12996, 11111], 64, 16, 72, None, 0),      # all of 16 rows
])
def test_four_heads_at_a_time(B, T, cap, lens, Hq, Hk, D, left, sinks, weighted):
    check(B, T, cap, lens, Hq, Hk, D, left, sinks, weighted)


def test_four_heads_at_a_time_over_a_tree():
    tree = words(63, 3, 3)
    check(3, 3, 5000, [4997, 0, 4000], 32, 32, 64, 4500, 4, True, tree)


@pytest.mark.parametrize("B,T,cap,Hq,Hk,D,left,sinks", [
    (70, 1, 500, 4, 2, 64, None, 0), (70, 1, 2500, 2, 1, 128, None, 0), (130, 3, 700, 4, 4, 64, 100, 5),
    (300, 1, 130, 2, 1, 64, None, 0), (300, 1, 1200, 1, 1, 64, None, 0), (65, 40, 300, 2, 1, 64, None, 0),
    (70, 40, 900, 1, 1, 128, 200, 3),
])
def test_many_samples(B, T, cap, Hq, Hk, D, left, sinks):
    lens = ramp(B, cap - T, B)
    check(B, T, cap, lens, Hq, Hk, D, left, sinks)
    check(B, T, cap, [0] * B, Hq, Hk, D, left, sinks, False)


@pytest.mark.parametrize("B,T,cap,lens,Hq,Hk,D", [
    (1, 1, 40000, [39999], 4, 1, 64),       # parts by the hundred
    (1, 2, 70000, [69000], 16, 1, 128),     # 32 rows
    (1, 33, 70000, [69900], 1, 1, 64),      # tiles of 128 rows, cut and joined with the weights
    (2, 33, 20000, [19000, 5], 4, 1, 128),  # 132 rows: tiles of 256
    (1, 400, 3000, [2600], 2, 2, 128),      # several tiles of rows a head
])
def test_parts_of_long_caches(B, T, cap, lens, Hq, Hk, D):
    check(B, T, cap, lens, Hq, Hk, D, None, 0)


@pytest.mark.parametrize("T,D", [(40, 128), (40, 64), (140, 128)])
def test_tiles_that_are_not_cut(T, D):
    """Enough rows for every compute unit: no parts, weights by their own pass."""
    check(16, T, 300, ramp(16, 300 - T, T), 32, 32, D, None, 0)


def test_scores_far_apart_over_the_parts():
    """A part whose maximum is far above or below the others', and slots that nothing
    is left for: exp(S - LSE) underflows there."""
    B, T, cap, Hq, Hk, D = 1, 1, 20000, 4, 1, 64
    q, k, v = rnd(64, B, T, Hq, D), rnd(65, B, cap, Hk, D), rnd(66, B, cap, Hk, D)
    k[:, 7000:7003] *= 40
    k[:, 15000:] *= 0.01
    for T in (1, 12):
        q = rnd(64, B, T, Hq, D)
        w = torch.rand((B, Hk, cap), device=DEV)
        o, lse, got = ut.cache_attn(q, k, v, dev([cap - T]), D ** -0.5, weights=w)
        check_attn(q, k, v, [cap - T], D ** -0.5, o, lse, None, None, 0, w, got)


def test_two_calls_at_once():
    """Calls on two streams, each with its own workspace: results as one by one."""
    sizes = ((2, 1, 9000, 8, 2, 128), (1, 48, 9000, 8, 2, 128), (1, 1, 3000, 4, 2, 64))
    calls = []
    for i, (B, T, cap, Hq, Hk, D) in enumerate(sizes):
        q, k, v = rnd(70 + i, B, T, Hq, D), rnd(80 + i, B, cap, Hk, D), rnd(90 + i, B, cap, Hk, D)
        lens, w = dev([cap - T] * B), torch.rand((B, Hk, cap), device=DEV)
        calls.append(lambda s=None, q=q, k=k, v=v, lens=lens, w=w, D=D: ut.cache_attn(
            q, k, v, lens, D ** -0.5, weights=w, stream=s))
    want = [c() for c in calls]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sizes]
    for turn in range(4):
        got = [c(s) for c, s in zip(calls, streams)]
        torch.cuda.synchronize()
        for a, b in zip(want, got):
            for x, y in zip(a, b):
                assert torch.equal(x, y)


def test_two_window_calls_at_once():
    qs = [draw(26 + i, 1, n, n, 4, 2, 64) for i, n in enumerate((3000, 1000))]
    want = [run(*x, 0.125, (60, 3), 200) for x in qs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in qs]
    for turn in range(3):
        got = [run(*x, 0.125, (60, 3), 200, stream=s) for x, s in zip(qs, streams)]
        torch.cuda.synchronize()
        for a, b in zip(want, got):
            for x, y in zip((a[0], a[1]) + a[2], (b[0], b[1]) + b[2]):
                assert torch.equal(x, y)


def test_graphs_with_a_workspace_of_both():
    """Two captured calls in one pool of memory, replayed in turn."""
    q, k, v = rnd(100, 2, 1, 8, 128), rnd(101, 2, 9000, 2, 128), rnd(102, 2, 9000, 2, 128)
    lens, w = dev([8000, 8999]), torch.rand((2, 2, 9000), device=DEV)
    x = draw(30, 1, 2000, 2000, 2, 2, 64)
    want = ut.cache_attn(q, k, v, lens, 0.1, weights=w)
    o, lse = ut.swattn_fwd(*x[:3], (60, 0), 0.125, 4)
    grads = ut.swattn_bwd(*x[:3], o, x[3], lse, (60, 0), 0.125, 4)
    torch.cuda.synchronize()
    one, two = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(one):
        got = ut.cache_attn(q, k, v, lens, 0.1, weights=w)
    with torch.cuda.graph(two, pool=one.pool()):
        got2 = ut.swattn_bwd(*x[:3], o, x[3], lse, (60, 0), 0.125, 4)
    for turn in range(4):
        (one if turn % 2 == 0 else two).replay()
        torch.cuda.synchronize()
        for a, b in zip(want if turn % 2 == 0 else grads, got if turn % 2 == 0 else got2):
            assert torch.equal(a, b)


@pytest.mark.parametrize("weighted", [False, True])
@pytest.mark.parametrize("B,T,cap,Hq,Hk", [(200, 1, 64, 1, 1), (2, 1, 300, 8, 2), (1, 1, 5000, 8, 2), (1, 40, 5000, 2, 1)])
def test_nothing_outside_the_workspace_is_written(B, T, cap, Hq, Hk, weighted):
    """Of many samples too short to be cut, whose workspace is none or the scores alone."""
    q, k, v = rnd(67, B, T, Hq, 64), rnd(68, B, cap, Hk, 64), rnd(69, B, cap, Hk, 64)
    lens = ramp(B, cap - T, 70)
    w = torch.rand((B, Hk, cap), device=DEV) if weighted else None
    got = torch.empty_like(w) if weighted else None
    need = ut.ut_cache_attn_workspace_size(B, T, cap, Hq, Hk, 64, with_weights=weighted)
    room = torch.full((need + 8192,), 91, dtype=torch.uint8, device=DEV)
    o, lse = torch.empty_like(q), torch.empty((B, Hq, T), device=DEV)
    assert ut.ut_cache_attn(q, k, v, o, lse, dev(lens), 0.125, weights_in=w, weights_out=got,
                            workspace=room[4096:4096 + need]) == ut.UT_OK
    torch.cuda.synchronize()
    assert (room[:4096] == 91).all() and (room[4096 + need:] == 91).all()
    check_attn(q, k, v, lens, 0.125, o, lse, None, None, 0, w, got)


# ---- validate mode ---------------------------------------------------------

def test_validate_mode_checks_the_lengths(monkeypatch):
    B, T, cap = 2, 3, 100
    q, k, v = rnd(110, B, T, 4, 64), rnd(111, B, cap, 2, 64), rnd(112, B, cap, 2, 64)
    w = torch.rand((B, 2, cap), device=DEV)
    monkeypatch.setenv("UT_VALIDATE", "1")
    _, lse, _ = ut.cache_attn(q, k, v, dev([97, 0]), 0.1, weights=w)
    ut.cache_weights(q, k, lse, dev([97, 0]), 0.1)
    ut.cache_evict(k, v, w, dev([100, 0]), 10)
    for bad in ([98, 0], [5, -1]):
        for call in (lambda: ut.cache_attn(q, k, v, dev(bad), 0.1, weights=w),
                     lambda: ut.cache_weights(q, k, lse, dev(bad), 0.1)):
            with pytest.raises(ut.UltraTexError) as e:
                call()
            assert e.value.status == ut.UT_ERR_INVALID_ARG
    for bad in ([101, 0], [5, -1]):
        with pytest.raises(ut.UltraTexError) as e:
            ut.cache_evict(k, v, w, dev(bad), 10)
        assert e.value.status == ut.UT_ERR_INVALID_ARG


def test_validate_mode_checks_the_windows_offsets(monkeypatch):
    g = torch.Generator().manual_seed(31)
    q, k, v, do = (torch.randn((100, 2, 64), generator=g).to(torch.bfloat16).to(DEV) for _ in range(4))
    good = offsets([50, 50])
    monkeypatch.setenv("UT_VALIDATE", "1")
    o, lse = ut.swattn_fwd_varlen(q, k, v, good, 50, good, 50, (9, 0), 0.125)
    ut.swattn_bwd_varlen(q, k, v, o, do, lse, good, 50, good, 50, (9, 0), 0.125)
    for at in ((offsets([50, 500]), 50, good, 50), (good, 49, good, 50), (good, 50, offsets([60, -3]), 60),
               (good, 50, good + 1, 50)):
        for call in (lambda: ut.swattn_fwd_varlen(q, k, v, *at, (9, 0), 0.125),
                     lambda: ut.swattn_bwd_varlen(q, k, v, o, do, lse, *at, (9, 0), 0.125)):
            with pytest.raises(ut.UltraTexError) as e:
                call()
            assert e.value.status == ut.UT_ERR_INVALID_ARG
