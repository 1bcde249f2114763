"""Cases for timing the position and cross-attention operators, beside their
plain forms.

Two operators of the multi-view transformer around the block-sparse attention:

* rotary positions with several axes (view, row, column) on the query and key
  rows that the attention reads, with the per-head RMS norm of queries and keys
  in front where the model has one (`qk_rope_fwd`, `qk_rope_bwd`);
* attention of the packed image tokens to an encoder's states of another
  length, forward and backward, for whole batches and for packed samples
  (`xattn_fwd`, `xattn_bwd`, `xattn_fwd_varlen`, `xattn_bwd_varlen`).

With `own` false `run` computes them from elementary torch operations in 32
bits (angles in 64); with `own` true it calls the library. `exact` computes the
same outputs in 64 bits.
"""
import math

import torch

own = False

DEV = "cuda"
THETA = 10000.0
EPS = 1e-6
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------

def listed():
    return [
        # queries and keys of a short text prompt: launches and host work
        {"name": "rope_prompt", "op": "rope", "n": 77, "hq": 8, "hk": 2, "dim": 64, "axes": "16,24,24",
         "views": 1, "rows": 7, "cols": 11, "kept": False, "norm": True, "pairs": "near", "type": "bf16",
         "train": False},
        # one layer of a denoising step, 2K canvas: kept tokens of 13 views
        {"name": "rope_step_2k", "op": "rope", "n": 77586, "hq": 24, "hk": 24, "dim": 128, "axes": "16,56,56",
         "views": 13, "rows": 128, "cols": 128, "kept": True, "norm": True, "pairs": "near", "type": "bf16",
         "train": False},
        # one training layer, 1K canvas, with the gradients of the norm's weights
        {"name": "rope_train_1k", "op": "rope", "n": 22879, "hq": 24, "hk": 24, "dim": 128, "axes": "16,56,56",
         "views": 13, "rows": 64, "cols": 64, "kept": True, "norm": True, "pairs": "near", "type": "bf16",
         "train": True},
        # frames of a video in fp32, two samples of one grid, no norm, odd sizes
        {"name": "rope_video_f32", "op": "rope", "n": 2 * 9 * 29 * 45, "hq": 10, "hk": 5, "dim": 72,
         "axes": "24,24,24", "views": 9, "rows": 29, "cols": 45, "kept": False, "norm": False, "pairs": "far",
         "type": "f32", "train": True},
        # the smallest training layer of the workloads against a short prompt
        {"name": "xattn_train_tiny", "op": "xattn", "batch": 1, "nq": 384, "nk": 77, "hq": 2, "hk": 2, "dim": 64,
         "short": 0.0, "train": True},
        # one query token a sample against long encoder states, shared key heads, padded
        {"name": "xattn_one_token", "op": "xattn", "batch": 4, "nq": 1, "nk": 16391, "hq": 32, "hk": 8, "dim": 128,
         "short": 0.3, "train": False},
        # one layer of a denoising step, 2K canvas, 512 text tokens
        {"name": "xattn_text_2k", "op": "xattn", "batch": 1, "nq": 77586, "nk": 512, "hq": 24, "hk": 24, "dim": 128,
         "short": 0.0, "train": False},
        # one training layer, 2K canvas, 512 text tokens
        {"name": "xattn_train_2k", "op": "xattn", "batch": 1, "nq": 77060, "nk": 512, "hq": 24, "hk": 24, "dim": 128,
         "short": 0.0, "train": True},
        # one layer of a denoising step, 1K canvas, against an image encoder's states
        {"name": "xattn_image_1k", "op": "xattn", "batch": 1, "nq": 22879, "nk": 4097, "hq": 24, "hk": 24, "dim": 128,
         "short": 0.0, "train": False},
        # a model with 64-wide heads in groups of four, padded encoder states
        {"name": "xattn_train_d64", "op": "xattn", "batch": 2, "nq": 9011, "nk": 1370, "hq": 16, "hk": 4, "dim": 64,
         "short": 0.4, "train": True},
        # eight samples of a 512-canvas bucket, each with its own prompt
        {"name": "xattn_train_packed", "op": "packed", "samples": 8, "qlo": 6011, "qhi": 6394, "klo": 17, "khi": 512,
         "hq": 24, "hk": 24, "dim": 128, "train": True},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rope", "xattn", "xattn", "packed"])
    hk = rng.choice([1, 2, 3, 5, 8, 12, 24])
    if op == "rope":
        views, rows, cols = rng.randint(1, 13), _log(rng, 4, 128), _log(rng, 4, 128)
        kept = rng.random() < 0.6
        cells = views * rows * cols
        n = max(1, int(cells * rng.uniform(0.05, 0.6))) if kept else cells * (rng.choice([1, 1, 2]) if cells < 30000 else 1)
        dim, axes = rng.choice([(32, "8,12,12"), (64, "16,24,24"), (64, "64"), (72, "24,24,24"), (96, "32,32,32"),
                                (128, "16,56,56"), (128, "32,32"), (256, "64,96,96")])
        hq = hk * rng.choice([1, 1, 2, 4])
        c = {"op": op, "n": n, "hq": hq, "hk": hk, "dim": dim, "axes": axes, "views": views, "rows": rows,
             "cols": cols, "kept": kept, "norm": rng.random() < 0.6, "pairs": rng.choice(["near", "far"]),
             "type": rng.choice(["bf16", "bf16", "f32"]), "train": rng.random() < 0.5}
        while work(c)["bytes"] > 1.9e9:
            group, c["hk"] = hq // hk, max(1, c["hk"] // 2)
            c["hq"], c["n"] = c["hk"] * group, c["n"] if c["hk"] > 1 or not kept else int(c["n"] * 0.7)
            if c["hk"] == 1:
                c["type"], c["train"] = "bf16", c["train"] and kept
        return c
    dim = rng.choice([64, 64, 128, 128, 128, 40, 80, 96])
    train = rng.random() < 0.6
    if op == "packed":
        qlo, klo = _log(rng, 1, 6000), _log(rng, 1, 600)
        c = {"op": op, "samples": rng.randint(1, 8), "qlo": qlo, "qhi": int(qlo * rng.uniform(1.0, 1.8)) + 1,
             "klo": klo, "khi": int(klo * rng.uniform(1.0, 4.0)) + 1, "hq": hk * rng.choice([1, 1, 2]), "hk": hk,
             "dim": dim, "train": train}
        while c["samples"] * c["qhi"] * c["hq"] * max(c["khi"], 250) > 4.5e8:
            c["qlo"], c["qhi"] = int(c["qlo"] * 0.7) + 1, int(c["qhi"] * 0.7) + 1
        return c
    c = {"op": op, "batch": rng.choice([1, 1, 2, 4]), "nq": _log(rng, 1, 77000), "nk": _log(rng, 1, 17000),
         "hq": hk * rng.choice([1, 1, 2, 4]), "hk": hk, "dim": dim, "short": rng.choice([0.0, 0.3, 0.7, 1.0]),
         "train": train}
    while c["batch"] * max(c["nq"], c["nk"]) * max(min(c["nq"], c["nk"]), 250) * c["hq"] > 4.5e8:
        k = "nq" if c["nq"] > c["nk"] else "nk"
        c[k] = int(c[k] * 0.7)
    return c


# ---------------------------------------------------------------------------
# inputs (plain torch, on the GPU, from the seed alone)
# ---------------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 7919 + 29)
    return g


def _normal(g, *shape, dtype=torch.bfloat16):
    return torch.randn(shape, generator=g, device=DEV, dtype=dtype)


def _axes(c):
    return tuple(int(a) for a in c["axes"].split(","))


def _spread(lo, hi, count):
    return [lo + (hi - lo) * i // max(count - 1, 1) for i in range(count)]


def _offsets(lens):
    return torch.tensor([0] + lens, device=DEV).cumsum(0).to(torch.int32)


def _places(lens):
    """Packed row of each padded place [B, longest], and padded place of each
    packed row; places behind a sample's end name a row of some sample."""
    longest, total = max(lens), sum(lens)
    start = torch.tensor([0] + lens[:-1]).cumsum(0)[:, None]
    j = torch.arange(longest)[None]
    live = j < torch.tensor(lens)[:, None]
    pad = (start + j).clamp(max=total - 1)
    flat = (torch.arange(len(lens))[:, None] * longest + j)[live]
    return pad.to(DEV), flat.to(DEV), live.to(DEV)


def _valid_lens(c):
    """Encoder states in use of each sample: all for the first, down to a share
    of 1 - short for the last (short = 1: the last has none, a dropped prompt)."""
    b = c["batch"]
    return [c["nk"] - int(round(c["short"] * c["nk"] * i / max(b - 1, 1))) for i in range(b)]


def prepare(case, seed):
    c, g = case, _gen(seed)
    st = {"case": c}
    hq, hk, d = c["hq"], c["hk"], c["dim"]
    if c["op"] == "rope":
        dt, n = DTYPES[c["type"]], c["n"]
        # queries and keys are views of the projection's output, values behind them
        proj = _normal(g, n, hq + 2 * hk, d, dtype=dt)
        cells = c["views"] * c["rows"] * c["cols"]
        i = torch.arange(cells, device=DEV)
        # grid coordinates; the last view is half as large in its own units
        pos = torch.stack([i // (c["rows"] * c["cols"]), i // c["cols"] % c["rows"], i % c["cols"]], 1).float()
        pos[i >= cells - c["rows"] * c["cols"], 1:] *= 0.5
        axes = _axes(c)
        st.update(q=proj[:, :hq], k=proj[:, hq:hq + hk], pos=pos[:, 3 - len(axes):].contiguous(), axes=axes,
                  idx=None, wq=None, wk=None)
        if c["kept"]:
            st["idx"] = torch.rand(cells, generator=g, device=DEV).argsort()[:n].sort().values.to(torch.int32)
        if c["norm"]:
            st["wq"], st["wk"] = ((1 + 0.2 * _normal(g, d, dtype=torch.float32)).to(dt) for _ in range(2))
        if c["train"]:
            st["dq"], st["dk"] = _normal(g, n, hq, d, dtype=dt), _normal(g, n, hk, d, dtype=dt)
        return st
    st["scale"] = 1.0 / math.sqrt(d)
    if c["op"] == "xattn":
        b, nq, nk = c["batch"], c["nq"], c["nk"]
        st["q"] = _normal(g, b, nq, hq, d)
        kv = _normal(g, b, nk, 2, hk, d)   # one projection of the encoder's states
        st["k"], st["v"] = kv[:, :, 0], kv[:, :, 1]
        st["mask"] = None
        if c["short"] > 0:
            lens = torch.tensor(_valid_lens(c), device=DEV)
            st["mask"] = (torch.arange(nk, device=DEV)[None] < lens[:, None]).to(torch.uint8)
    else:
        lq, lk = (_spread(c[a + "lo"], c[a + "hi"], c["samples"]) for a in ("q", "k"))
        st["q"] = _normal(g, sum(lq), hq, d)
        kv = _normal(g, sum(lk), 2, hk, d)
        st["k"], st["v"] = kv[:, 0], kv[:, 1]
        st.update(cuq=_offsets(lq), cuk=_offsets(lk), maxq=max(lq), maxk=max(lk), placeq=_places(lq),
                  placek=_places(lk))
    if c["train"]:
        st["do"] = torch.randn(st["q"].shape, generator=g, device=DEV, dtype=torch.bfloat16)
    return st


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(st):
    if own:
        return _run_own(st)
    c = st["case"]
    if c["op"] == "rope":
        return _plain_rope(st)
    if c["op"] == "xattn":
        return _plain_xattn(st)
    return _plain_packed(st)


def _run_own(st):
    import paper_2609_23169_amd as ut
    c = st["case"]
    if c["op"] == "rope":
        kw = {"theta": THETA, "token_idx": st["idx"], "q_weight": st["wq"], "k_weight": st["wk"], "eps": EPS,
              "interleaved": c["pairs"] == "near"}
        out = ut.qk_rope_fwd(st["q"], st["k"], st["pos"], st["axes"], **kw)
        if not c["train"]:
            return out
        if not c["norm"]:   # without the norm the gradient does not need the inputs
            return out + ut.qk_rope_bwd(st["dq"], st["dk"], st["pos"], st["axes"], **kw)[:2]
        return out + ut.qk_rope_bwd(st["dq"], st["dk"], st["pos"], st["axes"], q=st["q"], k=st["k"], **kw)
    if c["op"] == "xattn":
        o, lse = ut.xattn_fwd(st["q"], st["k"], st["v"], st["scale"], key_mask=st["mask"])
        if not c["train"]:
            return o, lse
        return (o, lse) + ut.xattn_bwd(st["q"], st["k"], st["v"], o, st["do"], lse, st["scale"],
                                       key_mask=st["mask"])
    at = (st["cuq"], st["maxq"], st["cuk"], st["maxk"])
    o, lse = ut.xattn_fwd_varlen(st["q"], st["k"], st["v"], *at, st["scale"])
    if not c["train"]:
        return o, lse
    return (o, lse) + ut.xattn_bwd_varlen(st["q"], st["k"], st["v"], o, st["do"], lse, *at, st["scale"])


# ---- plain forms ----------------------------------------------------------

def _turns(st):
    """cos and sin [n, 1, pairs] of every token: the angles in 64 bits."""
    n, pos = st["case"]["n"], st["pos"].double()
    at = st["idx"].long() if st["idx"] is not None else torch.arange(n, device=DEV) % pos.shape[0]
    parts = []
    for a, d in enumerate(st["axes"]):
        f = THETA ** (-torch.arange(0, d, 2, device=DEV, dtype=torch.float64) / d)
        parts.append(pos[at, a, None] * f)
    ang = torch.cat(parts, 1)[:, None]
    return ang.cos().float(), ang.sin().float()


def _rotate(x, cos, sin, pairs):
    r = 2 * cos.shape[-1]
    if pairs == "near":
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = x[..., :r // 2], x[..., r // 2:r]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([turned, x[..., r:]], -1)


def _plain_rope(st):
    c = st["case"]
    cos, sin = _turns(st)
    out, grads, wgrads = (), (), ()
    for x, w, dy in ((st["q"], st["wq"], st.get("dq")), (st["k"], st["wk"], st.get("dk"))):
        f = x.float()
        if c["norm"]:
            rstd = torch.rsqrt(f.square().mean(-1, keepdim=True) + EPS)
            hat = f * rstd
            f = hat * w.float()
        out += (_rotate(f, cos, sin, c["pairs"]).to(x.dtype),)
        if c["train"]:
            gr = _rotate(dy.float(), cos, -sin, c["pairs"])
            if c["norm"]:
                wgrads += ((gr * hat).sum((0, 1)),)
                gr = gr * w.float()
                gr = rstd * (gr - hat * (gr * hat).mean(-1, keepdim=True))
            grads += (gr.to(x.dtype),)
    return out + grads + wgrads


def _plain_attend(q, k, v, do, valid, scale):
    """q, do [B, Nq, Hq, D], k, v [B, Nk, Hk, D], valid [B, Nk] or None, in 32
    bits: (o, lse [B, Hq, Nq]) and, with do, (dq, dk, dv)."""
    b, nq, hq, d = q.shape
    hk = k.shape[2]

    def heads(x):   # [B, Hk, heads of the group x queries, D]
        return x.reshape(b, nq, hk, hq // hk, d).permute(0, 2, 3, 1, 4).reshape(b, hk, -1, d)

    def rows(x):
        return x.reshape(b, hk, hq // hk, nq, d).permute(0, 3, 1, 2, 4).reshape(b, nq, hq, d)

    qh, kh, vh = heads(q.float()), k.float().transpose(1, 2).contiguous(), v.float().transpose(1, 2).contiguous()
    s = torch.matmul(qh, kh.transpose(2, 3)) * scale
    if valid is not None:
        s = s.masked_fill(~valid[:, None, None], -math.inf)
    top = s.amax(3, keepdim=True)
    p = torch.exp(s - top.clamp(min=-1e30))
    total = p.sum(3, keepdim=True)
    lse = (top + total.log()).reshape(b, hq, nq)
    p = p / total.clamp(min=1e-30)
    o = torch.matmul(p, vh)
    if do is None:
        return (rows(o), lse)
    g = heads(do.float())
    ds = p * (torch.matmul(g, vh.transpose(2, 3)) - (g * o).sum(3, keepdim=True))
    dq = torch.matmul(ds, kh) * scale
    dk = torch.matmul(ds.transpose(2, 3), qh) * scale
    dv = torch.matmul(p.transpose(2, 3), g)
    return rows(o), lse, rows(dq), dk.transpose(1, 2), dv.transpose(1, 2)


def _plain_xattn(st):
    valid = st["mask"].bool() if st["mask"] is not None else None
    out = _plain_attend(st["q"], st["k"], st["v"], st.get("do"), valid, st["scale"])
    return tuple(x if i == 1 else x.to(torch.bfloat16).contiguous() for i, x in enumerate(out))


def _plain_packed(st):
    padq, flatq, liveq = st["placeq"]
    padk, flatk, livek = st["placek"]
    do = st["do"][padq] * liveq[:, :, None, None] if "do" in st else None
    out = _plain_attend(st["q"][padq], st["k"][padk], st["v"][padk], do, livek, st["scale"])

    def packed(x, flat):
        return x.flatten(0, 1)[flat].to(torch.bfloat16)

    o, lse = packed(out[0], flatq), out[1].transpose(0, 1).flatten(1)[:, flatq]
    if do is None:
        return o, lse
    return o, lse, packed(out[2], flatq), packed(out[3], flatk), packed(out[4], flatk)


# ---------------------------------------------------------------------------
# the work a pass cannot do without
# ---------------------------------------------------------------------------

def work(case):
    c = case
    hq, hk, d = c["hq"], c["hk"], c["dim"]
    if c["op"] == "rope":
        size = 2 if c["type"] == "bf16" else 4
        axes = _axes(c)
        elems = c["n"] * (hq + hk) * d
        # rows in and out; the gradient's rows in and out, with the norm the inputs are the forward's
        moved = elems * size * (4 if c["train"] else 2)
        table = c["views"] * c["rows"] * c["cols"] if not c["kept"] else c["n"]
        moved += 4 * (table * len(axes) + (c["n"] if c["kept"] else 0))
        per = 3 + (4 if c["norm"] else 0)
        return {"bytes": moved, "flops": elems * per * (2.5 if c["train"] else 1)}
    if c["op"] == "xattn":
        lq, lk = [c["nq"]] * c["batch"], _valid_lens(c)
    else:
        lq, lk = (_spread(c[a + "lo"], c[a + "hi"], c["samples"]) for a in ("q", "k"))
    pairs = sum(a * b for a, b in zip(lq, lk))
    rowq, rowk = sum(lq) * hq, sum(lk) * hk
    flops = 4.0 * pairs * hq * d
    # q, k, v in, o and lse out; for training dO in, dq, dk, dv out too
    moved = rowq * (2 * 2 * d + 4) + rowk * 2 * 2 * d
    if c["train"]:
        moved += rowq * 2 * 2 * d + rowk * 2 * 2 * d
        flops *= 3.5
    return {"bytes": moved, "flops": flops}


# ---------------------------------------------------------------------------
# the same results in 64 bits
# ---------------------------------------------------------------------------

def _exact_rope(c, st):
    n, d, axes = c["n"], c["dim"], _axes(c)
    row = torch.arange(n, device=DEV)
    row = row % st["pos"].shape[0] if st["idx"] is None else st["idx"].long()
    # pair p turns by place / theta^(2 i / axis size): unit complex numbers [n, pairs]
    unit = torch.cat([torch.exp(1j * (st["pos"][row, a].double()[:, None]
                                      / torch.pow(torch.tensor(THETA, dtype=torch.float64, device=DEV),
                                                  torch.arange(m // 2, device=DEV).double() * 2 / m)))
                      for a, m in enumerate(axes)], 1)
    m = unit.shape[1]
    if c["pairs"] == "near":
        first, second = torch.arange(m, device=DEV) * 2, torch.arange(m, device=DEV) * 2 + 1
    else:
        first, second = torch.arange(m, device=DEV), torch.arange(m, device=DEV) + m

    def turn(x, u):
        z = torch.complex(x[:, :, first], x[:, :, second]) * u[:, None]
        y = x.clone()
        y[:, :, first], y[:, :, second] = z.real, z.imag
        return y

    outs = {"q": [], "dq": [], "w": []}
    for x, w, dy in (("q", "wq", "dq"), ("k", "wk", "dk")):
        xd = st[x].double()
        if c["norm"]:
            wd = st[w].double()
            norm = ((xd * xd).sum(-1, keepdim=True) / d + EPS).sqrt()
            outs["q"].append(turn(xd / norm * wd, unit))
        else:
            outs["q"].append(turn(xd, unit))
        if not c["train"]:
            continue
        back = turn(st[dy].double(), unit.conj())
        if c["norm"]:
            outs["w"].append((back * xd / norm).sum(1).sum(0))
            back = back * wd
            back = back / norm - xd * (back * xd).sum(-1, keepdim=True) / (d * norm ** 3)
        outs["dq"].append(back)
    return tuple(outs["q"] + outs["dq"] + outs["w"])


def _exact_head(q, k, v, do, scale):
    """One head of one sample in 64 bits: [nq, d] queries on its [nk, d] states in use."""
    if k.shape[0] == 0:
        zero = torch.zeros_like(q)
        return zero, torch.full((q.shape[0],), -math.inf, dtype=torch.float64, device=DEV), zero, k, v
    s = (q @ k.T) * scale
    lse = torch.logsumexp(s, 1)
    p = torch.exp(s - lse[:, None])
    o = p @ v
    if do is None:
        return o, lse, None, None, None
    ds = p * (do @ v.T - (do * o).sum(1, keepdim=True))
    return o, lse, ds @ k * scale, ds.T @ q * scale, p.T @ do


def exact(case, seed):
    c = case
    st = prepare(c, seed)
    if c["op"] == "rope":
        return _exact_rope(c, st)
    hq, group = c["hq"], c["hq"] // c["hk"]
    if c["op"] == "xattn":
        lq, lk = [c["nq"]] * c["batch"], _valid_lens(c)
        atq = [(b, slice(None)) for b in range(c["batch"])]
        atk = [(b, slice(0, lk[b])) for b in range(c["batch"])]
        lse = torch.zeros((c["batch"], hq, c["nq"]), dtype=torch.float64, device=DEV)
    else:
        lq, lk = (_spread(c[a + "lo"], c[a + "hi"], c["samples"]) for a in ("q", "k"))
        endq, endk = ([0] + torch.tensor(x).cumsum(0).tolist() for x in (lq, lk))
        atq = [(slice(a, b),) for a, b in zip(endq, endq[1:])]
        atk = [(slice(a, b),) for a, b in zip(endk, endk[1:])]
        lse = torch.zeros((hq, sum(lq)), dtype=torch.float64, device=DEV)
    do = st.get("do")
    o, dq = (torch.zeros(st["q"].shape, dtype=torch.float64, device=DEV) for _ in range(2))
    dk, dv = (torch.zeros(st["k"].shape, dtype=torch.float64, device=DEV) for _ in range(2))
    for pq, pk in zip(atq, atk):
        for h in range(hq):
            got = _exact_head(st["q"][pq][:, h].double(), st["k"][pk][:, h // group].double(),
                              st["v"][pk][:, h // group].double(), do[pq][:, h].double() if do is not None else None,
                              st["scale"])
            o[pq][:, h] = got[0]
            if c["op"] == "xattn":
                lse[pq[0], h] = got[1]
            else:
                lse[h, pq[0]] = got[1]
            if do is not None and got[2] is not None:
                dq[pq][:, h] = got[2]
                if lk and got[3].shape[0]:
                    dk[pk][:, h // group] += got[3]
                    dv[pk][:, h // group] += got[4]
    return (o, lse) if do is None else (o, lse, dq, dk, dv)
