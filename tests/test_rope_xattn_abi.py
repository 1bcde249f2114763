"""Refusals of the rotary and cross-attention calls, on the host before any
launch (no GPU needed), and the binding's checks of tensors."""
import ctypes
import os
import subprocess
import sys

import pytest
import torch

import paper_2609_23169_amd as ut

FAKE = ctypes.c_void_p(0x10000)        # aligned, never dereferenced on these paths
ODD = ctypes.c_void_p(0x10004)         # 4-byte aligned only
I64, I32 = ctypes.c_int64, ctypes.c_int32


def _arr(t, xs):
    return None if xs is None else (t * len(xs))(*xs)


def _rope(fn="fwd", **kw):
    a = dict(q=FAKE, k=FAKE, q_out=FAKE, k_out=FAKE, dq=FAKE, dk=FAKE, strides=None, dtype=ut.UT_BF16, n=10, Hq=4,
             Hk=2, D=64, pos=FAKE, rows=10, idx=None, axes=(16, 24, 24), theta=10000.0, pairs=ut.UT_ROPE_NEAR,
             wq=FAKE, wk=FAKE, wd=ut.UT_BF16, eps=1e-6, dwq=FAKE, dwk=FAKE, ws=FAKE, wsb=1 << 24)
    a.update(kw)
    n_axes = a.get("n_axes", len(a["axes"]) if a["axes"] is not None else 1)
    mid = (_arr(I64, a["strides"]), a["dtype"], a["n"], a["Hq"], a["Hk"], a["D"], a["pos"], a["rows"], a["idx"],
           _arr(I32, a["axes"]), n_axes, a["theta"], a["pairs"], a["wq"], a["wk"], a["wd"], a["eps"])
    if fn == "fwd":
        return ut.lib().ut_qk_rope_fwd(a["q"], a["k"], a["q_out"], a["k_out"], *mid, None)
    return ut.lib().ut_qk_rope_bwd(a["q_out"], a["k_out"], a["q"], a["k"], a["dq"], a["dk"], *mid, a["dwq"], a["dwk"],
                                   a["ws"], a["wsb"], None)


BAD, UNS, WSP = ut.UT_ERR_INVALID_ARG, ut.UT_ERR_UNSUPPORTED, ut.UT_ERR_WORKSPACE


@pytest.mark.parametrize("fn", ["fwd", "bwd"])
@pytest.mark.parametrize("kw,status,msg", [
    (dict(n=-1), BAD, "n must be"), (dict(n=1 << 31), BAD, "n must be"),
    (dict(Hq=0), BAD, "Hq"), (dict(Hk=-1), BAD, "Hk"),
    (dict(D=60), UNS, "head_dim"), (dict(D=264), UNS, "head_dim"), (dict(D=0), UNS, "head_dim"),
    (dict(dtype=7), BAD, "dtype"), (dict(wd=7), BAD, "dtype"), (dict(pairs=2), BAD, "pair layout"),
    (dict(axes=None), BAD, "axes"), (dict(axes=(8,) * 5), BAD, "axes"), (dict(n_axes=0), BAD, "axes"),
    (dict(axes=(16, 23)), BAD, "even"), (dict(axes=(16, 0)), BAD, "even"), (dict(axes=(16, -2)), BAD, "even"),
    (dict(axes=(32, 34)), BAD, "axes take 66"), (dict(axes=(2147483646,) * 2), BAD, "axes take"),
    (dict(axes=(6, 6), pairs=ut.UT_ROPE_FAR), UNS, "multiple of 8"),
    (dict(theta=0.0), BAD, "theta"), (dict(theta=float("inf")), BAD, "theta"), (dict(theta=float("nan")), BAD, "theta"),
    (dict(rows=0), BAD, "pos_rows"), (dict(rows=1 << 31), BAD, "pos_rows"), (dict(pos=None), BAD, "pos is NULL"),
    (dict(wk=None), BAD, "both"), (dict(wq=None), BAD, "both"),
    (dict(eps=0.0), BAD, "eps"), (dict(eps=float("nan")), BAD, "eps"),
    (dict(q=None), BAD, "q is NULL"), (dict(q=ODD), BAD, "aligned"), (dict(k=None), BAD, "k is NULL"),
    (dict(q_out=None), BAD, "q_out is NULL"), (dict(k_out=ODD), BAD, "k_out must be 16-byte"),
    (dict(idx=ctypes.c_void_p(0x10001)), BAD, "token_idx"),
    (dict(strides=(248, 128, 256, 128, 256, 128)), BAD, "stride"),
    (dict(strides=(260, 128, 260, 128, 260, 128)), BAD, "stride"),
    (dict(strides=(1 << 31,) * 6), UNS, "stride"),
])
def test_rope_refusals(fn, kw, status, msg):
    assert _rope(fn, **kw) == status
    text = ut.last_error()
    assert text.startswith(f"ut_qk_rope_{fn}") and msg in text


def test_rope_strides_of_fp32_are_multiples_of_four():
    assert _rope(strides=(260, 132, 260, 132), dtype=ut.UT_F32, n=0) == ut.UT_OK
    assert _rope(strides=(258, 132, 260, 132), dtype=ut.UT_F32, n=0) == BAD


def test_rope_bwd_refuses_missing_gradients_and_workspace():
    need = ut.ut_qk_rope_bwd_workspace_size(64)
    assert need == 1024 * 2 * 64 * 4 and ut.ut_qk_rope_bwd_workspace_size(0) == 0
    assert ut.ut_qk_rope_bwd_workspace_size(257) == 0
    assert _rope("bwd", dwq=None) == BAD and "dq_weight" in ut.last_error()
    assert _rope("bwd", dwk=None) == BAD and "dk_weight" in ut.last_error()
    assert _rope("bwd", ws=None) == WSP and _rope("bwd", wsb=need - 1) == WSP
    assert _rope("bwd", ws=ODD) == BAD
    assert _rope("bwd", dq=None) == BAD and _rope("bwd", dk=None) == BAD


def test_rope_without_tokens_launches_nothing():
    assert _rope(n=0, q=None, k=None, q_out=None, k_out=None) == ut.UT_OK
    assert _rope("bwd", n=0, wq=None, wk=None, q=None, q_out=None, dq=None, ws=None, wsb=0) == ut.UT_OK


def _x(fn="fwd", varlen=False, **kw):
    a = dict(q=FAKE, k=FAKE, v=FAKE, o=FAKE, lse=FAKE, dout=FAKE, dq=FAKE, dk=FAKE, dv=FAKE, strides=None, mask=None,
             cuq=FAKE, cuk=FAKE, B=2, Tq=200, Tk=60, Nq=100, Nk=30, Hq=4, Hk=2, D=64, scale=0.1, ws=FAKE, wsb=1 << 40)
    a.update(kw)
    head = [a["q"], a["k"], a["v"], a["o"]]
    head += [a["lse"]] if fn == "fwd" else [a["dout"], a["lse"], a["dq"], a["dk"], a["dv"]]
    head += [_arr(I64, a["strides"]), a["mask"]]
    tail = [a["Hq"], a["Hk"], a["D"], a["scale"]]
    if varlen:
        head += [a["cuq"], a["cuk"], a["B"], a["Tq"], a["Tk"], a["Nq"], a["Nk"]] + tail + [1]
    else:
        head += [a["B"], a["Nq"], a["Nk"]] + tail
    return getattr(ut.lib(), f"ut_xattn_{fn}" + ("_varlen" if varlen else ""))(*head, a["ws"], a["wsb"], None)


@pytest.mark.parametrize("varlen", [False, True])
@pytest.mark.parametrize("fn", ["fwd", "bwd"])
@pytest.mark.parametrize("kw,status,msg", [
    (dict(B=0), BAD, "B"), (dict(Nq=-1), BAD, "lengths"), (dict(Nk=-1), BAD, "lengths"),
    (dict(Hq=0), BAD, "Hq"), (dict(Hk=0), BAD, "Hk"), (dict(Hq=5), BAD, "multiple of Hk"),
    (dict(D=0), UNS, "head_dim"), (dict(D=60), UNS, "head_dim"), (dict(D=136), UNS, "head_dim"),
    (dict(scale=0.0), BAD, "softmax_scale"), (dict(scale=-1.0), BAD, "softmax_scale"),
    (dict(scale=float("nan")), BAD, "softmax_scale"), (dict(scale=float("inf")), BAD, "softmax_scale"),
    (dict(B=65536, Nq=1024), BAD, "too large"), (dict(B=65536, Nk=2048), BAD, "too large"),
    (dict(q=None), BAD, "q is NULL"), (dict(k=ODD), BAD, "k must be 16-byte"), (dict(v=None), BAD, "v is NULL"),
    (dict(o=ODD), BAD, "o must be"), (dict(lse=None), BAD, "lse is NULL"),
    (dict(strides=(248,) + (256,) * 7), BAD, "stride of q"), (dict(strides=(260,) + (256,) * 7), BAD, "stride of q"),
    (dict(strides=(256, 1 << 22) + (256,) * 6), UNS, "stride of k"),
])
def test_xattn_refusals(fn, varlen, kw, status, msg):
    assert _x(fn, varlen, **kw) == status
    text = ut.last_error()
    assert text.startswith(f"ut_xattn_{fn}" + ("_varlen" if varlen else "")) and msg in text


@pytest.mark.parametrize("fn", ["fwd", "bwd"])
def test_xattn_varlen_refusals(fn):
    for kw, msg in ((dict(cuq=None), "cu_seqlens_q is NULL"), (dict(cuk=None), "cu_seqlens_k is NULL"),
                    (dict(Tq=-1), "outside"), (dict(Tk=1 << 31), "outside"), (dict(Tq=1 << 26), "too large")):
        assert _x(fn, True, **kw) == BAD
        assert msg in ut.last_error()


def test_xattn_workspaces():
    # few rows against many keys are split, everything else needs none
    assert ut.ut_xattn_fwd_workspace_size(1, 5000, 512, 24, 24, 128) == 0
    need = ut.ut_xattn_fwd_workspace_size(4, 1, 16384, 32, 8, 128)
    assert need > 0 and need % (4 * 32 * (128 * 4 + 8)) == 0
    size = dict(B=4, Nq=1, Nk=16384, Hq=32, Hk=8, D=128)
    assert _x(**size, wsb=need - 1) == WSP and _x(**size, ws=None) == WSP and _x(**size, ws=ODD) == BAD
    need = ut.ut_xattn_bwd_workspace_size(2, 100, 30, 4, 2, 64)
    assert need >= 2 * 100 * 4 * 8
    assert _x("bwd", wsb=need - 1) == WSP and _x("bwd", ws=None, wsb=0) == WSP
    for bad in ((0, 1, 1, 1, 1, 64), (1, -1, 1, 1, 1, 64), (1, 1, 1, 3, 2, 64), (1, 1, 1, 1, 1, 60)):
        assert ut.ut_xattn_fwd_workspace_size(*bad) == 0 and ut.ut_xattn_bwd_workspace_size(*bad) == 0
    assert ut.ut_xattn_fwd_varlen_workspace_size(0, 1, 1, 1, 1, 1, 64) == 0
    assert ut.ut_xattn_bwd_varlen_workspace_size(2, 200, 60, 100, 30, 4, 2, 64) == need


def test_xattn_without_queries_launches_nothing():
    assert _x(Nq=0, q=None, o=None, lse=None) == ut.UT_OK
    assert _x(varlen=True, Tq=0, q=None, o=None, lse=None) == ut.UT_OK
    assert _x("bwd", Nq=0, Nk=0, q=None, k=None, v=None, o=None, dout=None, lse=None, dq=None, dk=None, dv=None) == ut.UT_OK


# ---- the binding's checks (host tensors: refused before a launch) -----------

def _bf(*shape):
    return torch.zeros(shape, dtype=torch.bfloat16)


def test_binding_refuses_host_tensors_and_wrong_shapes():
    q, k, pos = _bf(6, 4, 64), _bf(6, 2, 64), torch.zeros(6, 3)
    ax = (16, 24, 24)
    for bad in (lambda: ut.qk_rope_fwd(q, k, pos, ax),                                    # host memory
                lambda: ut.qk_rope_fwd(q, _bf(6, 2, 32), pos, ax),                        # another head_dim
                lambda: ut.qk_rope_fwd(q, _bf(5, 2, 64), pos, ax),                        # another length
                lambda: ut.qk_rope_fwd(q, k.float(), pos, ax),                            # another dtype
                lambda: ut.qk_rope_fwd(q, k, pos.double(), ax),
                lambda: ut.qk_rope_fwd(q, k, pos, (16, 48)),                              # a column too many
                lambda: ut.qk_rope_fwd(q, k, pos, ax, token_idx=torch.zeros(6)),
                lambda: ut.qk_rope_fwd(q, k, pos, ax, token_idx=torch.zeros(5, dtype=torch.int32)),
                lambda: ut.qk_rope_fwd(q, k, pos, ax, q_weight=_bf(32), k_weight=_bf(64)),
                lambda: ut.qk_rope_fwd(q, k, pos, ax, q_weight=_bf(64), k_weight=torch.zeros(64)),
                lambda: ut.qk_rope_fwd(q.transpose(0, 1), None, pos, ax),                 # heads not contiguous
                lambda: ut.qk_rope_fwd(q[:1].expand(6, 4, 64), None, pos, ax),            # tokens overlap
                lambda: ut.qk_rope_bwd(q, k, pos, ax, q_weight=_bf(64), k_weight=_bf(64)),  # inputs missing
                lambda: ut.qk_rope_bwd(q, k, pos, ax, q=_bf(6, 2, 64))):
        with pytest.raises(ValueError):
            bad()
    q, k = _bf(2, 6, 4, 64), _bf(2, 5, 2, 64)
    lse = torch.zeros(2, 4, 6)
    for bad in (lambda: ut.xattn_fwd(q, k, k, 0.1), lambda: ut.xattn_fwd(q, k, _bf(2, 4, 2, 64), 0.1),
                lambda: ut.xattn_fwd(q, _bf(1, 5, 2, 64), _bf(1, 5, 2, 64), 0.1),
                lambda: ut.xattn_fwd(q.half(), k.half(), k.half(), 0.1),
                lambda: ut.xattn_fwd(q, k, k, 0.1, key_mask=torch.zeros(2, 5)),
                lambda: ut.xattn_fwd(q, k, k, 0.1, key_mask=torch.zeros(2, 6, dtype=torch.uint8)),
                lambda: ut.xattn_fwd(q[:, ::2][:, :2], k[:, :3], k[:, :3], 0.1),          # batches apart
                lambda: ut.xattn_bwd(q, k, k, q, q, lse.double(), 0.1),
                lambda: ut.xattn_bwd(q, k, k, q, q[:, :5], lse, 0.1)):
        with pytest.raises(ValueError):
            bad()
    q, k = _bf(12, 4, 64), _bf(10, 2, 64)
    cu = torch.tensor([0, 6, 12], dtype=torch.int32)
    for bad in (lambda: ut.xattn_fwd_varlen(q, k, k, cu, 6, cu[:2], 5, 0.1),
                lambda: ut.xattn_fwd_varlen(q, k, k, cu.long(), 6, cu, 5, 0.1),
                lambda: ut.xattn_fwd_varlen(q[None], k, k, cu, 6, cu, 5, 0.1)):
        with pytest.raises(ValueError):
            bad()


def test_token_stride_of_views():
    qkv = _bf(2, 7, 3, 4, 64)
    assert ut._token_stride(qkv[:, :, 1], "x") == 3 * 4 * 64
    assert ut._token_stride(qkv[0, :, 1], "x") == 3 * 4 * 64
    assert ut._token_stride(_bf(5, 4, 64)[::2], "x") == 2 * 4 * 64
    assert ut._token_stride(qkv[:1, :3, 0], "x") == 3 * 4 * 64       # one sample: any length
    for bad in (qkv[:, :5, 0], qkv[..., :32], qkv.permute(0, 1, 2, 4, 3)):
        with pytest.raises(ValueError):
            ut._token_stride(bad, "x")


@pytest.mark.parametrize("x,msg", [
    (_bf(1, 8, 64).expand(300, 8, 64), "tokens overlap"),              # one token for all
    (_bf(1, 1, 8, 64).expand(4, 1, 8, 64), "tokens overlap"),          # one learned query for the batch
    (_bf(1, 1, 4, 64).expand(1, 300, 4, 64), "tokens overlap"),        # the gradient of a sum over the tokens
    (_bf(2, 1, 4, 64).expand(2, 6, 4, 64), "tokens"),
    (_bf(1, 6, 4, 64).expand(2, 6, 4, 64), "evenly strided"),
    (_bf(1, 1, 64).expand(5, 1, 64), "tokens overlap"),                # a head of its own
    (_bf(7 * 128).as_strided((6, 4, 64), (128, 64, 1)), "tokens overlap"),
    (_bf(6, 1, 64).expand(6, 4, 64), "heads must be contiguous"),
    (_bf(4, 6, 64).transpose(0, 1), "heads must be contiguous"),
    (_bf(2, 6, 2, 64)[:, :3], "evenly strided"),
])
def test_token_stride_refuses(x, msg):
    """By their reason: rows that share memory would be read past their end."""
    with pytest.raises(ValueError, match=msg):
        ut._token_stride(x, "x")


def test_token_stride_of_the_gradient_of_a_sum():
    """As autograd hands it back: strides (256, 0, 64, 1) at one sample."""
    o = torch.zeros(1, 300, 4, 64, requires_grad=True)
    g, = torch.autograd.grad(o.sum(1), o, torch.ones(1, 4, 64))
    assert g.stride()[1] == 0
    with pytest.raises(ValueError, match="tokens overlap"):
        ut._token_stride(g, "dout")
    assert ut._token_stride(g.contiguous(), "dout") == 256
    assert ut._token_stride(torch.zeros(0, 4, 64), "x") == 256 == ut._token_stride(torch.zeros(1, 1, 4, 64), "x")


@pytest.mark.parametrize("varlen", [False, True])
@pytest.mark.parametrize("size", [dict(B=1 << 24, Nq=1, Nk=1, Hq=1, Hk=1), dict(B=1 << 21, Nq=1, Nk=7, Hq=8, Hk=8),
                                  dict(B=(1 << 24) - 7, Nq=1, Nk=3, Hq=1, Hk=1)])
def test_xattn_bwd_refuses_launches_of_too_many_workgroups(size, varlen):
    """The dK/dV pass has a workgroup of 256 threads a sample, key head and 128 keys; 2^24 of
    them are refused before anything is launched. The forward takes these sizes."""
    size = dict(size, D=8, Tq=size["B"], Tk=size["B"])
    n = [size["Hq"], size["Hk"], 8]
    query = (lambda s: ut.ut_xattn_bwd_varlen_workspace_size(s["B"], s["Tq"], s["Tk"], s["Nq"], s["Nk"], *n)) if varlen else (
        lambda s: ut.ut_xattn_bwd_workspace_size(s["B"], s["Nq"], s["Nk"], *n))
    assert query(size) == 0
    assert _x("bwd", varlen, **size) == BAD and "workgroups" in ut.last_error()
    assert _x("fwd", varlen, **size, q=None) == BAD and "q is NULL" in ut.last_error()
    less = dict(size, B=size["B"] - 1 if size["Hk"] > 1 else (1 << 24) - 8)
    assert query(less) > 0
    assert _x("bwd", varlen, **less, q=None) == BAD and "q is NULL" in ut.last_error()


def test_xattn_bwd_refuses_joins_of_too_many_rows():
    """Rows of few samples, split over keys, whose join would be a launch of 2^32 threads."""
    at = lambda t: (1, t, 64, 1, 100000, 1, 1, 128)  # noqa: E731
    assert ut.ut_xattn_bwd_varlen_workspace_size(*at((1 << 27) - 1)) == 0
    assert ut.ut_xattn_bwd_varlen_workspace_size(*at((1 << 27) - 8)) > 0


def test_validate_mode_without_host_memory_is_an_error():
    """Offsets of 2^31 - 1 samples take 8 GiB on the host: an error where there is less, no exception through the
    C entry. In a process of its own, with little address space and no HIP call before that."""
    code = """
import ctypes, resource
import paper_2609_23169_amd as ut
lib, fake = ut.lib(), ctypes.c_void_p(0x10000)
used = int(open("/proc/self/statm").read().split()[0]) * resource.getpagesize()
resource.setrlimit(resource.RLIMIT_AS, (used + (1 << 30),) * 2)
n = (1 << 31) - 1
for call, args in ((lib.ut_xattn_fwd_varlen, (*[fake] * 5, None, None, fake, fake, n, 10, 10, 0, 0, 1, 1, 64, 0.1, 0, None, 0, None)),
                   (lib.ut_bsattn_fwd_varlen, (*[fake] * 6, n, 10, 1, 1, 64, 64, fake, fake, 0.1, None))):
    st = call(*args)
    assert st == ut.UT_ERR_HIP and "memory" in ut.last_error(), (st, ut.last_error())
print("done")
"""
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=120,
                       cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                       env=dict(os.environ, UT_VALIDATE="1"))
    assert r.returncode == 0 and "done" in r.stdout, r.stderr[-2000:]


BIG = (1 << 32) + 6    # 6 in 32 bits


def test_sizes_past_32_bits_are_refused_not_cut():
    """The C calls take int32 sizes; larger ones must not arrive there as their low halves."""
    q, k, long_k = _bf(1, 6, 1, 64), _bf(1, 5, 1, 64), _bf(1, 1, 1, 64).expand(1, BIG, 1, 64)
    cu = torch.tensor([0, 6], dtype=torch.int32)
    pos = torch.zeros(6, 1)
    for call in (lambda: ut._xattn_args(q, long_k, long_k, None, 4), lambda: ut._xattn_args(long_k, k, k, None, 4),
                 lambda: ut._check_cu(cu, cu, BIG, 6), lambda: ut._check_cu(cu, cu, 6, BIG),
                 lambda: ut._check_cu(cu, cu, 6, -BIG),
                 lambda: ut._rope_args(q, None, pos, (BIG,), None, None, None),
                 lambda: ut._rope_args(q, None, pos, (-BIG,), None, None, None),
                 lambda: ut._rope_args(_bf(1, 1, 64).expand(1, BIG, 64), None, pos, (64,), None, None, None)):
        with pytest.raises(ValueError, match="32 bits"):
            call()
    for fn, args in ((ut.ut_xattn_fwd_workspace_size, (1, 1, 16384, 32, 8, 128)),
                     (ut.ut_xattn_bwd_workspace_size, (1, 600, 16384, 32, 8, 128)),
                     (ut.ut_xattn_fwd_varlen_workspace_size, (1, 1, 1, 16384, 32, 8, 128)),
                     (ut.ut_xattn_bwd_varlen_workspace_size, (1, 600, 600, 600, 16384, 32, 8, 128))):
        assert fn(*args) > 0
        for i in range(len(args)):
            assert fn(*args[:i], args[i] + (1 << 32), *args[i + 1:]) == 0, (fn.__name__, i)
    assert ut.ut_qk_rope_bwd_workspace_size(64 + (1 << 32)) == 0
