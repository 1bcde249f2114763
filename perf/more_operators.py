"""Cases for timing window attention, attention over a cache and eviction from
it, beside their plain forms.

Three operators for sequences whose keys stay for later queries:

* attention within a sliding window, with a few first tokens (sinks) that stay
  visible, forward and backward, for whole batches and packed samples
  (`swattn_fwd`, `swattn_bwd`, `swattn_fwd_varlen`, `swattn_bwd_varlen`);
* attention of single tokens, of chunks of a prompt and of trees of drafted
  tokens over a cache, with the attention weight that every slot has received
  (`cache_attn`);
* eviction from such a cache by that weight: selection and compaction
  (`cache_evict`).

Query i of Nq sits at position p = i + Nk - Nq of its sample's Nk keys and sees
key j where p - left <= j <= p + right, or j < sinks and (right > 0 or j <= p).

With `own` false `run` computes them from elementary torch operations in 32
bits; with `own` true it calls the library. `exact` computes the same outputs in
64 bits.
"""
import math

import torch

own = False

DEV = "cuda"


# ---------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------

def listed():
    return [
        # the smallest training layer of the workloads, causal
        {"name": "win_train_tiny", "op": "window", "batch": 1, "n": 384, "hq": 2, "hk": 2, "dim": 64, "left": 95,
         "right": 0, "sinks": 4, "short": 0.0, "train": True},
        # one layer of a denoising step, 2K canvas: local attention around every token, 512 text tokens in front
        {"name": "win_step_2k", "op": "window", "batch": 1, "n": 77586, "hq": 24, "hk": 24, "dim": 128, "left": 1024,
         "right": 1024, "sinks": 512, "short": 0.0, "train": False},
        # one training layer, 1K canvas, tokens generated in order
        {"name": "win_train_1k", "op": "window", "batch": 1, "n": 22879, "hq": 24, "hk": 24, "dim": 128, "left": 2047,
         "right": 0, "sinks": 4, "short": 0.0, "train": True},
        # a model with 64-wide heads in groups of four, padded samples
        {"name": "win_train_d64", "op": "window", "batch": 2, "n": 9011, "hq": 16, "hk": 4, "dim": 64, "left": 511,
         "right": 0, "sinks": 4, "short": 0.4, "train": True},
        # eight samples of a 512-canvas bucket, each with 77 text tokens in front
        {"name": "win_train_packed", "op": "packed", "samples": 8, "lo": 6011, "hi": 6394, "hq": 24, "hk": 24,
         "dim": 128, "left": 512, "right": 512, "sinks": 77, "train": True},
        # the next token of a short sequence: launches and host work
        {"name": "cache_short", "op": "cache", "batch": 1, "tokens": 1, "cap": 512, "low": 0.6, "hq": 8, "hk": 2,
         "dim": 64, "left": -1, "sinks": 0, "tree": False, "weights": True},
        # the next token of four long sequences, with the weights that eviction needs
        {"name": "cache_long", "op": "cache", "batch": 4, "tokens": 1, "cap": 16500, "low": 0.7, "hq": 32, "hk": 8,
         "dim": 128, "left": -1, "sinks": 0, "tree": False, "weights": True},
        # the next token of eight sequences that see a window of a long cache and its first tokens
        {"name": "cache_window", "op": "cache", "batch": 8, "tokens": 1, "cap": 24577, "low": 0.5, "hq": 32, "hk": 8,
         "dim": 128, "left": 4095, "sinks": 4, "tree": False, "weights": False},
        # 48 drafted tokens a sequence to be verified at once
        {"name": "cache_tree", "op": "cache", "batch": 4, "tokens": 48, "cap": 8300, "low": 0.6, "hq": 32, "hk": 8,
         "dim": 128, "left": -1, "sinks": 0, "tree": True, "weights": True},
        # a chunk of two prompts behind what the cache holds of them
        {"name": "cache_chunk", "op": "cache", "batch": 2, "tokens": 509, "cap": 11111, "low": 0.8, "hq": 24,
         "hk": 24, "dim": 128, "left": -1, "sinks": 0, "tree": False, "weights": False},
        # a short cache: launches and host work
        {"name": "evict_short", "op": "evict", "batch": 1, "cap": 300, "low": 1.0, "hk": 2, "dim": 64, "keep": 128,
         "sinks": 4, "recent": 32},
        # four long caches brought down to a quarter
        {"name": "evict_long", "op": "evict", "batch": 4, "cap": 16500, "low": 0.2, "hk": 8, "dim": 128, "keep": 4096,
         "sinks": 4, "recent": 1024},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["window", "window", "packed", "cache", "cache", "evict"])
    hk = rng.choice([1, 2, 3, 5, 8, 12, 24])
    dim = rng.choice([64, 64, 128, 128, 128, 40, 80, 96])
    if op in ("window", "packed"):
        left, causal = _log(rng, 16, 4000), rng.random() < 0.6
        c = {"op": op, "hq": hk * rng.choice([1, 1, 2, 4]), "hk": hk, "dim": dim, "left": left,
             "right": 0 if causal else rng.choice([left, _log(rng, 1, 2000)]),
             "sinks": rng.choice([0, 1, 4, 4, _log(rng, 5, 600)]), "train": rng.random() < 0.6}
        if op == "window":
            c.update(batch=rng.choice([1, 1, 2, 4]), n=_log(rng, 1, 40000), short=rng.choice([0.0, 0.0, 0.3, 0.8]))
        else:
            lo = _log(rng, 1, 6000)
            c.update(samples=rng.randint(1, 8), lo=lo, hi=int(lo * rng.uniform(1.0, 1.8)) + 1)
        while work(c)["flops"] > 1.9e12 or c["hq"] * sum(_lens(c)) > 600000:
            k = "n" if op == "window" else "hi"
            c[k] = int(c[k] * 0.7)
            if op == "packed":
                c["lo"] = min(c["lo"], c["hi"])
        return c
    c = {"op": op, "batch": rng.choice([1, 1, 2, 4, 8]), "hk": hk, "dim": dim, "low": rng.choice([0.0, 0.3, 0.7, 1.0])}
    if op == "evict":
        c["cap"] = _log(rng, 2, 60000)
        most = 50e6
    else:
        kind = rng.choice(["one", "one", "tree", "chunk"])
        t = 1 if kind == "one" else rng.randint(2, 64) if kind == "tree" else _log(rng, 2, 600)
        c.update(tokens=t, cap=t + _log(rng, 1, 30000), hq=hk * rng.choice([1, 1, 2, 4, 8]), tree=kind == "tree",
                 weights=kind != "chunk" and rng.random() < 0.6,
                 left=rng.choice([-1, -1, _log(rng, 64, 8000)]), sinks=rng.choice([0, 0, 4, 60]))
        most = 34e6
    while c["batch"] * c["cap"] * hk * dim > most or c["batch"] * c["cap"] * c.get("hq", 1) * c.get("tokens", 1) > 4e8:
        c["cap"] = max(int(c["cap"] * 0.7), c.get("tokens", 1) + 1)
        if c["cap"] == c.get("tokens", 1) + 1:
            c["batch"] = 1
            break
    if op == "evict":
        c["keep"] = max(1, int(c["cap"] * rng.uniform(0.05, 0.95)))
        c["sinks"] = min(c["keep"], rng.choice([0, 1, 4]))
        c["recent"] = int((c["keep"] - c["sinks"]) * rng.uniform(0.0, 0.6))
    return c


# ---------------------------------------------------------------------------
# inputs (plain torch, on the GPU, from the seed alone)
# ---------------------------------------------------------------------------

def _gen(seed, device=DEV):
    g = torch.Generator(device=device)
    g.manual_seed(int(seed) * 7919 + 31)
    return g


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.bfloat16)


def _spread(lo, hi, count):
    return [lo + (hi - lo) * i // max(count - 1, 1) for i in range(count)]


def _lens(c):
    """Tokens of every sample; of a cache the slots in use before the call."""
    if c["op"] == "window":
        return [c["n"]] * c["batch"]
    if c["op"] == "packed":
        return _spread(c["lo"], c["hi"], c["samples"])
    full = c["cap"] - c.get("tokens", 0)
    return _spread(int(round(full * c["low"])), full, c["batch"])[::-1]


def _used(c):
    """Keys of every sample of a padded batch that are in use."""
    b = c["batch"]
    return [c["n"] - int(round(c["short"] * c["n"] * i / max(b - 1, 1))) for i in range(b)]


def _trees(seed, batch, tokens):
    """For each drafted token the drafted tokens that it sees, a bit each: itself
    and its ancestors. Token 0 is the root; later ones continue an earlier one."""
    g = _gen(seed, "cpu")
    pick = torch.rand((batch, tokens), generator=g).tolist()
    rows = []
    for b in range(batch):
        seen = [1]
        for t in range(1, tokens):
            seen.append(seen[int(t * math.sqrt(pick[b][t]))] | 1 << t)
        rows.append([s - (1 << 64) if s >= 1 << 63 else s for s in seen])
    return torch.tensor(rows, dtype=torch.int64, device=DEV)


def prepare(case, seed):
    c, g = case, _gen(seed)
    st = {"case": c}
    hk, d = c["hk"], c["dim"]
    if c["op"] in ("window", "packed"):
        lens = _lens(c)
        shape = (c["batch"], c["n"]) if c["op"] == "window" else (sum(lens),)
        # queries, keys and values are views of one projection's output
        proj = _normal(g, *shape, c["hq"] + 2 * hk, d)
        st["q"], st["k"], st["v"] = proj[..., :c["hq"], :], proj[..., c["hq"]:c["hq"] + hk, :], proj[..., c["hq"] + hk:, :]
        st["mask"] = None
        if c["op"] == "packed":
            st["cu"] = torch.tensor([0] + lens, device=DEV).cumsum(0).to(torch.int32)
            st["longest"] = max(lens)
        elif c["short"] > 0:
            used = torch.tensor(_used(c), device=DEV)
            st["mask"] = (torch.arange(c["n"], device=DEV)[None] < used[:, None]).to(torch.uint8)
        if c["train"]:
            st["do"] = _normal(g, *shape, c["hq"], d)
        st["scale"] = 1.0 / math.sqrt(d)
        return st
    b, cap = c["batch"], c["cap"]
    st["len"] = torch.tensor(_lens(c), device=DEV, dtype=torch.int32)
    st["k"], st["v"] = _normal(g, b, cap, hk, d), _normal(g, b, cap, hk, d)
    # what the slots have received so far: few much, most little, some nothing at all
    w = torch.exp(2.0 * torch.randn((b, hk, cap), generator=g, device=DEV)) * 0.1
    w = w * (torch.rand((b, hk, cap), generator=g, device=DEV) > 0.05)
    st["weights"] = w * (torch.arange(cap, device=DEV) < st["len"][:, None, None])
    if c["op"] == "cache":
        st["q"] = _normal(g, b, c["tokens"], c["hq"], d)
        st["tree"] = _trees(seed, b, c["tokens"]) if c["tree"] else None
        st["scale"] = 1.0 / math.sqrt(d)
    return st


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(st):
    if own:
        return _run_own(st)
    return {"window": _plain_window, "packed": _plain_packed, "cache": _plain_cache,
            "evict": _plain_evict}[st["case"]["op"]](st)


def _run_own(st):
    import paper_2609_23169_amd as ut
    c = st["case"]
    if c["op"] == "window":
        kw = {"n_sink": c["sinks"], "key_mask": st["mask"]}
        at = ((c["left"], c["right"]), st["scale"])
        o, lse = ut.swattn_fwd(st["q"], st["k"], st["v"], *at, **kw)
        if not c["train"]:
            return o, lse
        return (o, lse) + ut.swattn_bwd(st["q"], st["k"], st["v"], o, st["do"], lse, *at, **kw)
    if c["op"] == "packed":
        at = (st["cu"], st["longest"], st["cu"], st["longest"], (c["left"], c["right"]), st["scale"])
        o, lse = ut.swattn_fwd_varlen(st["q"], st["k"], st["v"], *at, n_sink=c["sinks"])
        if not c["train"]:
            return o, lse
        return (o, lse) + ut.swattn_bwd_varlen(st["q"], st["k"], st["v"], o, st["do"], lse, *at, n_sink=c["sinks"])
    if c["op"] == "cache":
        return ut.cache_attn(st["q"], st["k"], st["v"], st["len"], st["scale"], tree=st["tree"],
                             window_left=c["left"] if c["left"] >= 0 else None, n_sink=c["sinks"],
                             weights=st["weights"] if c["weights"] else None)
    return ut.cache_evict(st["k"], st["v"], st["weights"], st["len"], c["keep"], n_sink=c["sinks"],
                          n_recent=c["recent"])


# ---- plain forms ----------------------------------------------------------

CHUNK = 1024


def _plain_band(q, k, v, do, used, c, scale):
    """One sample, q, do [n, Hq, D], k, v [n, Hk, D], used [n] or None, in 32 bits: (o,
    lse [Hq, n]) and, with do, (dq, dk, dv). Queries in chunks, each with the
    sinks and the keys of its windows."""
    n, hq, d = q.shape
    hk = k.shape[1]
    group = hq // hk
    qh = q.float().transpose(0, 1)
    kh, vh = (x.float().transpose(0, 1) for x in (k, v))
    dh = do.float().transpose(0, 1) if do is not None else None
    o, lse = torch.zeros_like(qh), torch.zeros((hq, n), device=DEV)
    if do is not None:
        dq, dk, dv = torch.zeros_like(qh), torch.zeros_like(kh), torch.zeros_like(vh)
    for a in range(0, n, CHUNK):
        z = min(a + CHUNK, n)
        lo, hi = max(0, a - c["left"]), min(n, z + c["right"])
        first = min(c["sinks"], lo if c["right"] > 0 else min(lo, z))
        later = min(c["sinks"], n) if c["right"] > 0 else hi
        parts = [(0, first), (lo, hi), (max(hi, 0), max(later, hi))]
        at = torch.cat([torch.arange(x, y, device=DEV) for x, y in parts])
        p = torch.arange(a, z, device=DEV)[:, None]
        see = ((at >= p - c["left"]) & (at <= p + c["right"])) | (
            (at < c["sinks"]) & ((at <= p) if c["right"] == 0 else (at >= 0)))
        if used is not None:
            see = see & used[at]
        kc, vc = kh[:, at], vh[:, at]
        kc, vc = (x.repeat_interleave(group, 0) for x in (kc, vc))
        s = torch.matmul(qh[:, a:z], kc.transpose(1, 2)) * scale
        s = s.masked_fill(~see, -math.inf)
        top = s.amax(2, keepdim=True)
        e = torch.exp(s - top.clamp(min=-1e30))
        total = e.sum(2, keepdim=True)
        lse[:, a:z] = (top + total.log())[..., 0]
        e = e / total.clamp(min=1e-30)
        o[:, a:z] = torch.matmul(e, vc)
        if do is None:
            continue
        g = dh[:, a:z]
        ds = e * (torch.matmul(g, vc.transpose(1, 2)) - (g * o[:, a:z]).sum(2, keepdim=True))
        dq[:, a:z] = torch.matmul(ds, kc) * scale
        dk[:, at] += torch.matmul(ds.transpose(1, 2), qh[:, a:z]).unflatten(0, (hk, group)).sum(1) * scale
        dv[:, at] += torch.matmul(e.transpose(1, 2), g).unflatten(0, (hk, group)).sum(1)
    out = (o.transpose(0, 1), lse)
    if do is not None:
        out += (dq.transpose(0, 1), dk.transpose(0, 1), dv.transpose(0, 1))
    return out


def _plain_window(st):
    c = st["case"]
    per = []
    for b in range(c["batch"]):
        used = st["mask"][b].bool() if st["mask"] is not None else None
        per.append(_plain_band(st["q"][b], st["k"][b], st["v"][b], st["do"][b] if c["train"] else None, used, c,
                               st["scale"]))
    return tuple(torch.stack(x) if i == 1 else torch.stack(x).to(torch.bfloat16) for i, x in enumerate(zip(*per)))


def _plain_packed(st):
    c, per, at = st["case"], [], 0
    for n in _lens(c):
        s = slice(at, at + n)
        per.append(_plain_band(st["q"][s], st["k"][s], st["v"][s], st["do"][s] if c["train"] else None, None, c,
                               st["scale"]))
        at += n
    return tuple(torch.cat(x, 1) if i == 1 else torch.cat(x, 0).to(torch.bfloat16) for i, x in enumerate(zip(*per)))


def _bits(words, count):
    """Bits 0 .. count - 1 of int64 words, [..., count] truth values."""
    return (words[..., None] >> torch.arange(count, device=DEV)) & 1 != 0


def _plain_cache(st):
    c = st["case"]
    b, t, hq, d = st["q"].shape
    cap, hk = c["cap"], c["hk"]
    length = st["len"].long()[:, None, None]
    slot = torch.arange(cap, device=DEV)[None, None]
    if c["tree"]:
        seen = _bits(st["tree"], t)                                       # [B, T, T]
        own_bit = torch.eye(t, dtype=torch.bool, device=DEV)
        place = length + (seen & ~own_bit).sum(2, keepdim=True)
        drafted = slot - length
        in_tree = (drafted >= 0) & (drafted < t)
        in_tree = in_tree & torch.gather(seen, 2, drafted.clamp(0, t - 1).expand(b, t, cap))
        see = (slot < length) | in_tree
    else:
        place = length + torch.arange(t, device=DEV)[None, :, None]
        see = slot <= place
    if c["left"] >= 0:
        see = see & ((slot >= place - c["left"]) | (slot < c["sinks"]) | (c["tree"] & (slot >= length)))
    qh = st["q"].float().reshape(b, t, hk, hq // hk, d).permute(0, 2, 3, 1, 4).reshape(b, hk, -1, d)
    kh, vh = (x.float().transpose(1, 2) for x in (st["k"], st["v"]))
    s = torch.matmul(qh, kh.transpose(2, 3).contiguous()) * st["scale"]
    see = see[:, None].repeat(1, 1, hq // hk, 1)                          # rows: heads of the group x tokens
    s = s.masked_fill(~see, -math.inf)
    top = s.amax(3, keepdim=True)
    e = torch.exp(s - top.clamp(min=-1e30))
    total = e.sum(3, keepdim=True)
    lse = (top + total.log()).reshape(b, hq, t)
    e = e / total.clamp(min=1e-30)
    vh = vh.masked_fill((slot >= length + t)[..., None], 0.0)
    o = torch.matmul(e, vh.contiguous())
    o = o.reshape(b, hk, hq // hk, t, d).permute(0, 3, 1, 2, 4).reshape(b, t, hq, d).to(torch.bfloat16)
    if not c["weights"]:
        return o, lse
    return o, lse, st["weights"] + e.sum(2)


def _plain_evict(st):
    c = st["case"]
    b, cap, hk, d = st["k"].shape
    keep = c["keep"]
    length = st["len"].long()[:, None]
    slot = torch.arange(cap, device=DEV)[None]
    w = st["weights"]
    rank = w.masked_fill(((slot < c["sinks"]) | (slot >= length - c["recent"]))[:, None], math.inf)
    rank = rank.masked_fill((slot >= length)[:, None], -math.inf)
    best = rank.sort(dim=2, descending=True, stable=True).indices[:, :, :keep]
    count = length.clamp(max=keep)
    place = torch.arange(keep, device=DEV)
    live = (place < count)[:, None].expand(b, hk, keep)
    # slots not in use sort last; those of a short cache are ended by its length
    idx = best.masked_fill(~live, cap).sort(2).values
    at = idx.clamp(max=cap - 1)
    row = at.transpose(1, 2)[..., None].expand(b, keep, hk, d)
    dead = ~live.transpose(1, 2)[..., None]
    k, v = (torch.gather(st[x], 1, row).masked_fill(dead, 0) for x in ("k", "v"))
    return (k, v, torch.gather(w, 2, at).masked_fill(~live, 0), count[:, 0].to(torch.int32),
            idx.masked_fill(~live, -1).to(torch.int32))


# ---------------------------------------------------------------------------
# the work a pass cannot do without
# ---------------------------------------------------------------------------

def _pairs(n, used, c):
    """Visible pairs of one sample of n tokens, the first `used` keys in use, and
    its keys that are visible to some query."""
    left, right, sinks = c["left"], c["right"], min(c["sinks"], used)
    p = torch.arange(n)
    lo = (p - left).clamp(min=0)
    hi = (p + right).clamp(max=used - 1)
    inside = (hi - lo + 1).clamp(min=0)
    end = p.clamp(max=sinks - 1) + 1 if right == 0 else torch.full((n,), sinks)
    before = torch.minimum(end, lo)
    after = (end - (hi + 1).clamp(min=0)).clamp(min=0) if right > 0 else 0
    return int((inside + before + after).sum())


def work(case):
    c = case
    hk, d = c["hk"], c["dim"]
    if c["op"] == "evict":
        lens = _lens(c)
        kept = sum(min(n, c["keep"]) for n in lens)
        rows = c["batch"] * c["keep"] * hk
        # weights of the slots in use, kept rows; rows, weights and slots out
        return {"bytes": hk * (sum(lens) * 4 + kept * 2 * 2 * d) + rows * (2 * 2 * d + 8), "flops": hk * sum(lens)}
    hq = c["hq"]
    if c["op"] == "cache":
        t, pairs, keys = c["tokens"], 0, 0
        for n in _lens(c):
            ctx = n if c["left"] < 0 else min(n, c["left"] + min(c["sinks"], max(n - c["left"], 0)))
            pairs += t * ctx + t * (t + 1) // 2
            keys += min(n + t, ctx + t)
        moved = c["batch"] * t * hq * (2 * 2 * d + 4) + keys * hk * 2 * 2 * d
        if c["weights"]:
            moved += 2 * 4 * c["batch"] * hk * c["cap"]
        return {"bytes": moved, "flops": 4.0 * pairs * hq * d}
    lens = _lens(c)
    used = _used(c) if c["op"] == "window" else lens
    pairs = sum(_pairs(n, u, c) for n, u in zip(lens, used))
    rowq, rowk = sum(lens) * hq, sum(used) * hk
    flops = 4.0 * pairs * hq * d
    moved = rowq * (2 * 2 * d + 4) + rowk * 2 * 2 * d
    if c["train"]:   # dO in, dq, dk, dv out too
        moved += rowq * 2 * 2 * d + sum(lens) * hk * 2 * 2 * d
        flops *= 3.5
    return {"bytes": moved, "flops": flops}


# ---------------------------------------------------------------------------
# the same results in 64 bits
# ---------------------------------------------------------------------------

def _attend64(q, k, v, do, see, scale):
    """One head's rows [n, d] on keys [m, d], see [n, m], in 64 bits."""
    s = (q @ k.T * scale).where(see, torch.tensor(-math.inf, dtype=torch.float64, device=DEV))
    lse = torch.logsumexp(s, 1)
    p = torch.exp(s - lse[:, None]).where(see, torch.zeros((), dtype=torch.float64, device=DEV))
    o = p @ v
    if do is None:
        return o, lse, p, None, None, None
    ds = p * ((do @ v.T) - (do * o).sum(1)[:, None])
    return o, lse, p, ds @ k * scale, ds.T @ q * scale, p.T @ do


def _exact_sample(q, k, v, do, used, c, scale):
    n, hq, d = q.shape
    group = hq // k.shape[1]
    o, dq = (torch.zeros((n, hq, d), dtype=torch.float64, device=DEV) for _ in range(2))
    dk, dv = (torch.zeros(k.shape, dtype=torch.float64, device=DEV) for _ in range(2))
    lse = torch.zeros((hq, n), dtype=torch.float64, device=DEV)
    j = torch.arange(n, device=DEV)
    for a in range(0, n, 4096):
        i = j[a:a + 4096, None]
        far = (j - i > c["right"]) | (i - j > c["left"])
        see = ~far | ((j < c["sinks"]) & (j <= (i if c["right"] == 0 else n)))
        see &= j < used
        keys = see.any(0).nonzero()[:, 0]
        see, rows = see[:, keys], i[:, 0]
        for h in range(hq):
            x = h // group
            got = _attend64(q[rows, h].double(), k[keys, x].double(), v[keys, x].double(),
                            do[rows, h].double() if do is not None else None, see, scale)
            o[rows, h], lse[h, rows] = got[0], got[1]
            if do is not None:
                dq[rows, h] = got[3]
                dk[keys, x] += got[4]
                dv[keys, x] += got[5]
    return (o, lse) if do is None else (o, lse, dq, dk, dv)


def _exact_cache(c, st):
    b, t, hq, d = st["q"].shape
    group = hq // c["hk"]
    o = torch.zeros(st["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.zeros((b, hq, t), dtype=torch.float64, device=DEV)
    weights = st["weights"].double()
    for x in range(b):
        n = _lens(c)[x]
        see = torch.zeros((t, n + t), dtype=torch.bool)
        for i in range(t):
            if c["tree"]:
                word = int(st["tree"][x, i])
                seen = [u for u in range(t) if word >> u & 1]
                depth = sum(u != i for u in seen)
                see[i, [n + u for u in seen]] = True
            else:
                depth = i
                see[i, n:n + i + 1] = True
            first = 0 if c["left"] < 0 else max(0, n + depth - c["left"])
            see[i, first:n] = True
            if first > n and not c["tree"]:
                see[i, n:first] = False
            see[i, :min(c["sinks"], n + i + 1 if not c["tree"] else n)] = True
        see = see.to(DEV)
        for h in range(hq):
            kd, vd = (st[y][x, :n + t, h // group].double() for y in ("k", "v"))
            got = _attend64(st["q"][x, :, h].double(), kd, vd, None, see, st["scale"])
            o[x, :, h], lse[x, h] = got[0], got[1]
            weights[x, h // group, :n + t] += got[2].sum(0)
    return (o, lse, weights) if c["weights"] else (o, lse)


def _exact_evict(c, st):
    b, cap, hk, d = st["k"].shape
    keep = c["keep"]
    k, v = (torch.zeros((b, keep, hk, d), dtype=torch.float64, device=DEV) for _ in range(2))
    w = torch.zeros((b, hk, keep), dtype=torch.float64, device=DEV)
    slots = torch.full((b, hk, keep), -1, dtype=torch.int32, device=DEV)
    counts = []
    for x, n in enumerate(_lens(c)):
        counts.append(min(n, keep))
        for h in range(hk):
            if n <= keep:
                at = list(range(n))
            else:
                a, z = c["sinks"], n - c["recent"]
                free = keep - c["sinks"] - c["recent"]
                value = st["weights"][x, h, a:z].tolist()
                best = sorted(range(z - a), key=lambda i: (-value[i], i))[:free]
                at = list(range(a)) + sorted(a + i for i in best) + list(range(z, n))
            at = torch.tensor(at, dtype=torch.int64, device=DEV)
            m = at.numel()
            k[x, :m, h], v[x, :m, h] = st["k"][x, at, h].double(), st["v"][x, at, h].double()
            w[x, h, :m] = st["weights"][x, h, at].double()
            slots[x, h, :m] = at.to(torch.int32)
    return k, v, w, torch.tensor(counts, dtype=torch.int32, device=DEV), slots


def exact(case, seed):
    c = case
    st = prepare(c, seed)
    if c["op"] == "evict":
        return _exact_evict(c, st)
    if c["op"] == "cache":
        return _exact_cache(c, st)
    per, at = [], 0
    for x, n in enumerate(_lens(c)):
        s = x if c["op"] == "window" else slice(at, at + n)
        at += n
        per.append(_exact_sample(st["q"][s], st["k"][s], st["v"][s], st["do"][s] if c["train"] else None,
                                 _used(c)[x] if c["op"] == "window" else n, c, st["scale"]))
    join = torch.stack if c["op"] == "window" else torch.cat
    return tuple(torch.cat(x, 1) if i == 1 and c["op"] == "packed" else join(x) for i, x in enumerate(zip(*per)))
