"""Refusals of the window-attention and cache calls, on the host before any launch
(no GPU needed), their workspaces, and the binding's checks of tensors."""
import ctypes

import pytest
import torch

import paper_2609_23169_amd as ut

FAKE = ctypes.c_void_p(0x10000)        # aligned, never dereferenced on these paths
ODD = ctypes.c_void_p(0x10004)         # 4-byte aligned only
BYTE = ctypes.c_void_p(0x10001)
I64 = ctypes.c_int64
BAD, UNS, WSP = ut.UT_ERR_INVALID_ARG, ut.UT_ERR_UNSUPPORTED, ut.UT_ERR_WORKSPACE


def _strides(xs):
    return None if xs is None else (I64 * len(xs))(*xs)


def _sw(fn="fwd", varlen=False, **kw):
    a = dict(q=FAKE, k=FAKE, v=FAKE, o=FAKE, lse=FAKE, dout=FAKE, dq=FAKE, dk=FAKE, dv=FAKE, strides=None, mask=None,
             cuq=FAKE, cuk=FAKE, B=2, Tq=200, Tk=200, Nq=100, Nk=100, Hq=4, Hk=2, D=64, left=30, right=0, sinks=4,
             scale=0.1, ws=FAKE, wsb=1 << 40)
    a.update(kw)
    head = [a["q"], a["k"], a["v"], a["o"]]
    head += [a["lse"]] if fn == "fwd" else [a["dout"], a["lse"], a["dq"], a["dk"], a["dv"]]
    head += [_strides(a["strides"]), a["mask"]]
    tail = [a["Hq"], a["Hk"], a["D"], a["left"], a["right"], a["sinks"], a["scale"]]
    if varlen:
        head += [a["cuq"], a["cuk"], a["B"], a["Tq"], a["Tk"], a["Nq"], a["Nk"]] + tail + [1]
    else:
        head += [a["B"], a["Nq"], a["Nk"]] + tail
    return getattr(ut.lib(), f"ut_swattn_{fn}" + ("_varlen" if varlen else ""))(*head, a["ws"], a["wsb"], None)


@pytest.mark.parametrize("varlen", [False, True])
@pytest.mark.parametrize("fn", ["fwd", "bwd"])
@pytest.mark.parametrize("kw,status,msg", [
    (dict(left=-2), BAD, "window"), (dict(right=-2), BAD, "window"), (dict(sinks=-1), BAD, "n_sink"),
    (dict(B=0), BAD, "B"), (dict(Nq=-1), BAD, "lengths"), (dict(Hq=5), BAD, "multiple of Hk"),
    (dict(D=60), UNS, "head_dim"), (dict(D=136), UNS, "head_dim"), (dict(scale=0.0), BAD, "softmax_scale"),
    (dict(scale=float("nan")), BAD, "softmax_scale"), (dict(B=65536, Nq=1024), BAD, "too large"),
    (dict(q=None), BAD, "q is NULL"), (dict(k=ODD), BAD, "k must be 16-byte"), (dict(lse=None), BAD, "lse is NULL"),
    (dict(strides=(248,) + (256,) * 7), BAD, "stride of q"), (dict(strides=(256, 1 << 22) + (256,) * 6), UNS, "stride of k"),
])
def test_swattn_refusals(fn, varlen, kw, status, msg):
    assert _sw(fn, varlen, **kw) == status
    text = ut.last_error()
    assert text.startswith(f"ut_swattn_{fn}" + ("_varlen" if varlen else "")) and msg in text


@pytest.mark.parametrize("fn", ["fwd", "bwd"])
def test_swattn_varlen_refusals(fn):
    for kw, msg in ((dict(cuq=None), "cu_seqlens_q is NULL"), (dict(cuk=None), "cu_seqlens_k is NULL"),
                    (dict(Tq=-1), "outside"), (dict(Tk=1 << 31), "outside"), (dict(Tq=1 << 26), "too large")):
        assert _sw(fn, True, **kw) == BAD
        assert msg in ut.last_error()


def test_swattn_workspaces():
    # many rows: no split of the keys; one row on a long window: split
    assert ut.ut_swattn_fwd_workspace_size(1, 20000, 20000, 24, 24, 128, (1024, 0), 4) == 0
    need = ut.ut_swattn_fwd_workspace_size(4, 1, 16384, 32, 8, 128, (None, 0), 0)
    assert need > 0 and need % (4 * 32 * (128 * 4 + 8)) == 0
    # a short window has few tiles, whatever the length
    assert ut.ut_swattn_fwd_workspace_size(4, 1, 16384, 32, 8, 128, (100, 0), 4) == 0
    size = dict(B=4, Nq=1, Nk=16384, Hq=32, Hk=8, D=128, left=-1)
    assert _sw(**size, wsb=need - 1) == WSP and _sw(**size, ws=None) == WSP and _sw(**size, ws=ODD) == BAD
    need = ut.ut_swattn_bwd_workspace_size(2, 100, 100, 4, 2, 64, (30, 0), 4)
    assert need >= 2 * 100 * 4 * 8
    assert _sw("bwd", wsb=need - 1) == WSP and _sw("bwd", ws=None, wsb=0) == WSP
    # sinks that most of a long sequence sees take partial sums, of that part alone
    plain = ut.ut_swattn_bwd_workspace_size(1, 77060, 77060, 24, 24, 128, (1024, 1024), 0)
    sinks = ut.ut_swattn_bwd_workspace_size(1, 77060, 77060, 24, 24, 128, (1024, 1024), 4)
    assert 0 < sinks - plain <= 64 * 128 * 24 * 128 * 8
    for bad in ((0, 1, 1, 1, 1, 64), (1, -1, 1, 1, 1, 64), (1, 1, 1, 3, 2, 64), (1, 1, 1, 1, 1, 60)):
        assert ut.ut_swattn_fwd_workspace_size(*bad, (1, 0)) == 0 and ut.ut_swattn_bwd_workspace_size(*bad, (1, 0)) == 0
    assert ut.lib().ut_swattn_bwd_workspace_size(1, 10, 10, 1, 1, 64, -2, 0, 0) == 0
    assert ut.lib().ut_swattn_fwd_workspace_size(1, 1, 10000, 1, 1, 64, 0, 0, -1) == 0
    assert ut.last_error() == ""
    # extreme windows and sinks overflow nothing
    big = (1 << 31) - 1
    assert ut.ut_swattn_fwd_workspace_size(4, 1, 16384, 32, 8, 128, (big, big), big) == \
        ut.ut_swattn_fwd_workspace_size(4, 1, 16384, 32, 8, 128, (None, None), 0)


def _ca(fn="attn", **kw):
    a = dict(q=FAKE, k=FAKE, v=FAKE, o=FAKE, lse=FAKE, strides=None, lens=FAKE, tree=None, tokens=None, win=None,
             wout=None, B=2, T=3, cap=300, Hq=4, Hk=2, D=64, left=-1, sinks=0, scale=0.1, ws=FAKE, wsb=1 << 40)
    a.update(kw)
    sizes = [a[x] for x in ("B", "T", "cap", "Hq", "Hk", "D", "left", "sinks", "scale")]
    if fn == "attn":
        return ut.lib().ut_cache_attn(a["q"], a["k"], a["v"], a["o"], a["lse"], _strides(a["strides"]), a["lens"],
                                      a["tree"], a["win"], a["wout"], *sizes, a["ws"], a["wsb"], None)
    return ut.lib().ut_cache_weights(a["q"], a["k"], a["lse"], _strides(a["strides"]), a["lens"], a["tree"],
                                     a["tokens"], a["win"], a["wout"], *sizes, None)


@pytest.mark.parametrize("fn", ["attn", "weights"])
@pytest.mark.parametrize("kw,status,msg", [
    (dict(T=0), BAD, "T must"), (dict(T=301), BAD, "T must"), (dict(cap=0), BAD, "T must"), (dict(B=0), BAD, "B"),
    (dict(Hq=3), BAD, "multiple of Hk"), (dict(D=12), UNS, "head_dim"), (dict(left=-2), BAD, "window"),
    (dict(sinks=-1), BAD, "n_sink"), (dict(scale=-1.0), BAD, "softmax_scale"),
    (dict(T=65, tree=FAKE), BAD, "at most 64"), (dict(T=9, tree=FAKE, left=7), BAD, "window must hold"),
    (dict(tree=ODD), BAD, "tree must be 8-byte"), (dict(lens=None), BAD, "cache_len is NULL"),
    (dict(lens=BYTE), BAD, "cache_len must be"), (dict(q=None), BAD, "q is NULL"), (dict(k=ODD), BAD, "must be 16-byte"),
    (dict(lse=None), BAD, "lse is NULL"), (dict(win=FAKE), BAD, "weights_out"), (dict(wout=BYTE), BAD, "weights_out must"),
    (dict(win=BYTE, wout=FAKE), BAD, "weights_in must"), (dict(strides=(256, 120, 128, 256)), BAD, "stride"),
    (dict(B=1 << 20, cap=300), BAD, "too large"),
])
def test_cache_refusals(fn, kw, status, msg):
    if fn == "weights" and kw == dict(strides=(256, 120, 128, 256)):
        kw = dict(strides=(256, 120))
    if fn == "weights":
        kw = dict({"wout": FAKE}, **kw)
        if kw.get("win") is FAKE:
            kw["wout"] = None
    assert _ca(fn, **kw) == status, ut.last_error()
    text = ut.last_error()
    assert text.startswith(f"ut_cache_{fn}") and msg in text


def test_cache_weights_refusals():
    assert _ca("weights") == BAD and "weights_out is NULL" in ut.last_error()
    assert _ca("weights", wout=FAKE, T=65, tokens=FAKE) == BAD and "at most 64" in ut.last_error()
    assert _ca("weights", wout=FAKE, tokens=ODD) == BAD and "tokens must be 8-byte" in ut.last_error()


@pytest.mark.parametrize("fn", ["attn", "weights"])
def test_weights_in_and_out_lie_apart_or_are_one(fn):
    n = 2 * 2 * 300 * 4
    for by in (4, n - 4, -4, 4 - n):
        assert _ca(fn, win=0x10000000, wout=0x10000000 + by, lens=None) == BAD
        assert "weights_out overlaps weights_in" in ut.last_error()
    for by in (0, n, -n):   # accepted: the next refusal
        assert _ca(fn, win=0x10000000, wout=0x10000000 + by, lens=None) == BAD and "cache_len is NULL" in ut.last_error()


def test_cache_workspaces():
    need = ut.ut_cache_attn_workspace_size(4, 1, 16500, 32, 8, 128)
    assert need > 0
    assert ut.ut_cache_attn_workspace_size(4, 1, 16500, 32, 8, 128, 100, 4) == 0
    assert ut.ut_cache_attn_workspace_size(4, 0, 16500, 32, 8, 128) == 0
    assert ut.ut_cache_attn_workspace_size(4, 16501, 16500, 32, 8, 128) == 0
    size = dict(B=4, T=1, cap=16500, Hq=32, Hk=8, D=128)
    assert _ca(**size, wsb=need - 1) == WSP and _ca(**size, ws=None) == WSP and _ca(**size, ws=ODD) == BAD


def _ev(**kw):
    p = lambda i: ctypes.c_void_p(0x10000000 * i)  # noqa: E731
    a = dict(k=p(1), v=p(2), w=p(3), lens=p(4), ko=p(5), vo=p(6), wo=p(7), lo=p(8), idx=p(9), strides=None, B=2, cap=300,
             capo=100, Hk=2, D=64, keep=100, sinks=4, recent=20, zero=1)
    a.update(kw)
    return ut.lib().ut_cache_evict(*(a[x] for x in ("k", "v", "w", "lens", "ko", "vo", "wo", "lo", "idx")),
                                   _strides(a["strides"]), *(a[x] for x in ("B", "cap", "capo", "Hk", "D", "keep", "sinks",
                                                                            "recent", "zero")), None)


@pytest.mark.parametrize("kw,status,msg", [
    (dict(B=0), BAD, "B in"), (dict(B=65536), BAD, "B in"), (dict(Hk=0), BAD, "Hk"), (dict(cap=0), BAD, "capacity"),
    (dict(keep=0), BAD, "n_keep"), (dict(keep=101), BAD, "n_keep"), (dict(sinks=-1), BAD, "n_sink"),
    (dict(recent=-1), BAD, "n_sink"), (dict(sinks=90, recent=11), BAD, "at most n_keep"),
    (dict(sinks=(1 << 31) - 1, recent=(1 << 31) - 1), BAD, "at most n_keep"), (dict(D=60), UNS, "head_dim"),
    (dict(D=136), UNS, "head_dim"), (dict(cap=1 << 25), BAD, "too large"), (dict(capo=1 << 25), BAD, "too large"),
    (dict(k=None), BAD, "k_cache is NULL"), (dict(v=ODD), BAD, "v_cache must be 16-byte"), (dict(ko=None), BAD, "k_out"),
    (dict(vo=ODD), BAD, "v_out must"), (dict(w=None), BAD, "weights is NULL"), (dict(wo=BYTE), BAD, "weights_out must"),
    (dict(lens=None), BAD, "cache_len"), (dict(lo=None), BAD, "len_out"), (dict(idx=BYTE), BAD, "kept_idx"),
    (dict(strides=(120, 128, 128, 128)), BAD, "stride of k_cache"), (dict(strides=(128, 128, 128, 1 << 22)), UNS, "stride"),
])
def test_evict_refusals(kw, status, msg):
    assert _ev(**kw) == status, ut.last_error()
    text = ut.last_error()
    assert text.startswith("ut_cache_evict") and msg in text


def test_evict_refuses_overlap():
    k, row = 0x10000000, 2 * 64 * 2          # bytes of a slot
    size = 2 * 300 * row
    at = ctypes.c_void_p
    assert _ev(ko=at(k)) == BAD and "k_out overlaps k_cache" in ut.last_error()
    assert _ev(vo=at(k + size - 16)) == BAD and "v_out overlaps k_cache" in ut.last_error()
    assert _ev(ko=at(0x20000000 - 2 * 100 * row + 16)) == BAD and "k_out overlaps v_cache" in ut.last_error()
    assert _ev(wo=at(0x30000000)) == BAD and "weights_out overlaps weights" in ut.last_error()
    assert _ev(lo=at(0x40000004)) == BAD and "len_out overlaps cache_len" in ut.last_error()


def test_the_binding_checks_tensors():
    q, kv = torch.zeros(2, 3, 4, 64, dtype=torch.bfloat16), torch.zeros(2, 9, 2, 64, dtype=torch.bfloat16)
    lens = torch.zeros(2, dtype=torch.int32)
    lse = torch.zeros(2, 4, 3)
    with pytest.raises(ValueError):   # host memory
        ut.swattn_fwd(q, kv, kv, (3, 0), 0.1)
    for window in ((-2, 0), (3, -5), (1 << 31, 0)):
        with pytest.raises(ValueError):
            ut.swattn_fwd(q, kv, kv, window, 0.1)
    for kw in (dict(cache_len=lens.long()), dict(cache_len=lens[:1]), dict(tree=torch.zeros(2, 3)),
               dict(tree=torch.zeros(2, 4, dtype=torch.int64)), dict(weights=torch.zeros(2, 2, 8)),
               dict(weights=torch.zeros(2, 2, 9, dtype=torch.float64)), dict(window_left=-3)):
        with pytest.raises(ValueError):
            ut.cache_attn(q, kv, kv, **dict(dict(cache_len=lens, softmax_scale=0.1), **kw))
    with pytest.raises(ValueError):
        ut.cache_weights(q, kv, lse, lens, 0.1, tokens=torch.zeros(3, dtype=torch.int64))
    w = torch.zeros(2, 2, 9)
    for args, kw in (((kv, kv[:1], w, lens, 4), {}), ((kv, kv, w[:, :1], lens, 4), {}), ((kv, kv.float(), w, lens, 4), {}),
                     ((kv, kv, w, lens.long(), 4), {}), ((kv, kv, w, lens, 1 << 31), dict(capacity=4))):
        with pytest.raises((ValueError, RuntimeError)):
            ut.cache_evict(*args, **kw)

