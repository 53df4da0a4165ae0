"""The two ends of a language model, timed alone: the embedding of its tokens and the loss over its vocabulary.

Both in the form in which the library carries every tensor, a pair: the mean m
and the half difference d over the two points theta +- eps v.

* embed: rows of the table for a batch of tokens, times a scale, with learned
  positions added for the GPT-2 family (fwd), and the gradients of the tables
  from that of the rows (bwd): one sum per token of the vocabulary;
* head: the softmax cross-entropy of x W^T against a target per row,
  without logits that stay: the loss of every row (loss), and with it the
  gradients of x and of W (grad).

``run`` without ``own`` is the plain form: products of pairs,
(a b).m = a.m b.m + a.d b.d and (a b).d = a.m b.d + a.d b.m, in elementary
torch operations in float32, sums over tokens in float64.  ``exact`` evaluates
the operators at the two points in float64 instead and takes the mean and the
half difference of the results.
"""
import math

import torch

own = False

EPS = 1e-3
IGNORE = -100       # a target that is left out

# Vocabularies and widths of the workloads.
TINY = dict(V=256, d=64, dtype="f32")
SMALL = dict(V=8192, d=512, dtype="f32")
MEDIUM = dict(V=32000, d=1024, dtype="bf16")
M1B = dict(V=32000, d=2048, dtype="bf16")
M8B = dict(V=128256, d=4096, dtype="bf16")


def listed():
    return [
        # one token of the 1.3B shape: launch latency
        dict(M1B, name="embed fwd one token", op="embed_fwd", B=1, S=1, scale=1.0, pos=False, pad=0),
        # the 1.3B workload's batch, scaled by the root of the width
        dict(M1B, name="embed fwd 1.3B", op="embed_fwd", B=4, S=2048, scale=math.sqrt(2048.0), pos=False, pad=0),
        # learned positions, odd lengths, rows inside a wider buffer
        dict(MEDIUM, name="embed fwd positions", op="embed_fwd", B=7, S=1001, scale=1.0, pos=True, pad=8),
        # the 1.3B workload's batch, backward: a quarter of the table's rows get a sum
        dict(M1B, name="embed bwd 1.3B", op="embed_bwd", B=4, S=2048, scale=math.sqrt(2048.0), pos=False, pad=0),
        # a long batch over a small vocabulary: sums of thousands of rows, positions too
        dict(SMALL, name="embed bwd long fp32", op="embed_bwd", B=65, S=509, scale=1.0, pos=True, pad=0),
        # the largest table: nearly all of it is zeros
        dict(M8B, name="embed bwd 8B", op="embed_bwd", B=1, S=2048, scale=64.0, pos=False, pad=0),
        # the loss of one token of the 1.3B shape: the table is read once
        dict(M1B, name="head loss one token", op="head_loss", T=1, ignore=0.0, pad=0),
        # scoring a padded batch, no gradients
        dict(MEDIUM, name="head loss padded", op="head_loss", T=2500, ignore=0.3, pad=0),
        # the tiny workload's batch, latency of loss and gradients
        dict(TINY, name="head grad tiny fp32", op="head_grad", T=512, ignore=0.0, pad=0),
        # an odd number of rows inside a wider buffer, fp32
        dict(SMALL, name="head grad odd fp32", op="head_grad", T=2047, ignore=0.1, pad=12),
        # the 1.3B workload's batch
        dict(M1B, name="head grad 1.3B", op="head_grad", T=8192, ignore=0.0, pad=0),
        # the largest: the vocabulary of the 8B workload, its batch
        dict(M8B, name="head grad 8B", op="head_grad", T=2048, ignore=0.1, pad=0),
    ]


def _log_between(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["embed_fwd", "embed_bwd", "head_loss", "head_grad", "head_grad"])
    c = dict(op=op, dtype=rng.choice(["bf16", "bf16", "f32"]))
    c["V"] = 8 * _log_between(rng, 8, 16032)
    c["d"] = 8 * _log_between(rng, 8, 512)
    c["pad"] = rng.choice([0, 0, 4, 8 * rng.randint(1, 16)])
    rows = _log_between(rng, 1, 32768 if op.startswith("embed") else 16384)
    if op.startswith("embed"):
        c["B"] = rng.randint(1, min(65, rows))
        c["S"] = max(1, rows // c["B"])
        c["scale"] = rng.choice([1.0, math.sqrt(c["d"]), rng.uniform(0.5, 50.0)])
        c["pos"] = rng.random() < 0.4
        while work(c)["bytes"] > 2.1e9 and c["V"] > 64:      # just below the largest listed table
            c["V"] = c["V"] // 16 * 8
        while work(c)["bytes"] > 2.1e9 and c["S"] > 1:
            c["S"] = (c["S"] + 1) // 2
    else:
        if c["dtype"] == "bf16":
            c["pad"] = c["pad"] // 8 * 8
        c["T"] = rows
        c["ignore"] = rng.choice([0.0, 0.1, 0.5])
        cap = 1.0e12 if c["dtype"] == "bf16" else 2.0e11     # T V d, just below the largest listed
        while c["T"] * c["V"] * c["d"] > cap and c["T"] > 1:
            c["T"] = (c["T"] + 1) // 2
    return c


def _dt(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _zipf(g, V, n):
    """Token ids with frequencies that fall as a power of their rank."""
    w = torch.arange(1, V + 1, device="cuda", dtype=torch.float64) ** -1.1
    cdf = torch.cumsum(w / w.sum(), 0)
    u = torch.rand(n, device="cuda", dtype=torch.float64, generator=g)
    return torch.searchsorted(cdf, u).clamp_(max=V - 1).to(torch.int32)


def _inputs(c, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    V, d, dt = c["V"], c["d"], _dt(c)

    def randn(*shape):
        return torch.randn(shape, device="cuda", generator=g)

    def rows(T, dtype, scales):
        # columns of unequal scale, as a residual stream has them
        col = torch.exp(0.5 * randn(d)) / math.exp(0.25)
        out = []
        for s in scales:
            full = torch.zeros((T, d + c["pad"]), device="cuda", dtype=dtype)
            full[:, :d] = (randn(T, d) * (s * col)).to(dtype)
            out.append(full[:, :d])
        return tuple(out)

    st = dict(case=c)
    if c["op"].startswith("embed"):
        st["tok"] = _zipf(g, V, c["B"] * c["S"]).view(c["B"], c["S"])
        if c["op"] == "embed_fwd":
            st["table"] = ((0.02 * randn(V, d)).to(dt), randn(V, d))
            st["table_pos"] = ((0.02 * randn(c["S"], d)).to(dt), randn(c["S"], d)) if c["pos"] else None
        else:
            st["dx"] = rows(c["B"] * c["S"], torch.float32, (1e-4 * EPS,))[0]
    else:
        T = c["T"]
        # normed rows and logits of a few units, half differences about EPS below
        st["x"] = rows(T, dt, (1.0, EPS))
        w = randn(V, d) * (2.0 / math.sqrt(d))
        st["w"] = (w.to(dt), (EPS * (2.0 / math.sqrt(d)) * randn(V, d)).to(dt))
        tgt = _zipf(g, V, T)
        tgt[torch.rand(T, device="cuda", generator=g) < c["ignore"]] = IGNORE
        st["tgt"] = tgt
        st["scale"] = 1.0 / T
    return st


def prepare(case, seed):
    st = _inputs(case, seed)
    if own:
        from paper_2602_00816_amd import fdhvp as fd

        c = case
        V, d, dev = c["V"], c["d"], "cuda"
        if c["op"].startswith("embed"):
            m = fd.Model("gpt2" if c["pos"] else "llama", 0, d, 1, 1, 8, V, max(2, c["S"]), c["dtype"],
                         embed_scale=c["scale"])
            if c["op"] == "embed_fwd":
                full = [torch.zeros((c["B"] * c["S"], d + c["pad"]), device=dev) for _ in range(2)]
                st["out"] = tuple(t[:, :d] for t in full)
            else:
                st["out"] = torch.empty((V, d), device=dev)
                st["out_pos"] = torch.empty((max(2, c["S"]), d), device=dev) if c["pos"] else None
                st["scratch"] = m.embed_scratch(c["B"], c["S"])
        else:
            m = fd.Model("llama", 0, d, 1, 1, 8, V, 2, c["dtype"])
            st["loss"] = tuple(torch.empty(c["T"], device=dev) for _ in range(2))
            st["scratch"] = m.head_scratch(c["T"], grads=c["op"] == "head_grad")
            if c["op"] == "head_grad":
                st["dx"] = tuple(torch.empty((c["T"], d), device=dev, dtype=_dt(c)) for _ in range(2))
                st["dw"] = torch.empty((V, d), device=dev, dtype=_dt(c))
        st["model"] = m
    return st


def run(state):
    c = state["case"]
    if own:
        m = state["model"]
        if c["op"] == "embed_fwd":
            return m.embed_forward(state["tok"], state["table"], eps=EPS, positions=state["table_pos"], out=state["out"])
        if c["op"] == "embed_bwd":
            r = m.embed_backward(state["dx"], state["tok"], eps=EPS, out=state["out"], out_positions=state["out_pos"],
                                 scratch=state["scratch"])
            return (r[0], r[1][:c["S"]]) if c["pos"] else r
        if c["op"] == "head_loss":
            return m.head_loss(state["x"], state["w"], state["tgt"], out=state["loss"], scratch=state["scratch"])
        return m.head_grad(state["x"], state["w"], state["tgt"], scale=state["scale"], eps=EPS, loss=state["loss"],
                           dx=state["dx"], dw=state["dw"], scratch=state["scratch"])
    return {"embed_fwd": _plain_embed, "embed_bwd": _plain_embed_grad}.get(c["op"], _plain_head)(state)


# ---- the plain form ---------------------------------------------------------------
def _plain_embed(state):
    c = state["case"]
    tok = state["tok"].long()
    e, ve = state["table"]
    m, d = c["scale"] * e[tok].float(), (c["scale"] * EPS) * ve[tok]
    if c["pos"]:
        p, vp = state["table_pos"]
        m, d = m + p.float(), d + EPS * vp
    return m.flatten(0, 1), d.flatten(0, 1)


def _plain_embed_grad(state):
    c = state["case"]
    dx = state["dx"].double()
    e = torch.zeros((c["V"], c["d"]), device="cuda", dtype=torch.float64)
    e.index_add_(0, state["tok"].flatten().long(), dx)
    e = (e * (c["scale"] / EPS)).float()
    if not c["pos"]:
        return e
    return e, (dx.view(c["B"], c["S"], -1).sum(0) / EPS).float()


def _plain_head(state):
    c = state["case"]
    dt = _dt(c)
    xm, xd = (t.float() for t in state["x"])
    wm, wd = (t.float() for t in state["w"])
    lm = xm @ wm.T + xd @ wd.T
    ld = xd @ wm.T + xm @ wd.T
    top = lm.amax(1, keepdim=True)
    e = torch.exp(lm - top)
    a, b = e * torch.cosh(ld), e * torch.sinh(ld)
    zm, zd = a.sum(1, keepdim=True), b.sum(1, keepdim=True)
    zz = (zm + zd) * (zm - zd)
    keep = state["tgt"] != IGNORE
    y = torch.where(keep, state["tgt"], 0).long()[:, None]
    loss_m = top + 0.5 * torch.log(zz) - lm.gather(1, y)
    loss_d = torch.atanh(zd / zm) - ld.gather(1, y)
    loss = tuple(torch.where(keep, t[:, 0], 0.0) for t in (loss_m, loss_d))
    if c["op"] == "head_loss":
        return loss
    g = (state["scale"] * keep.float())[:, None]
    pm, pd = (a * zm - b * zd) / zz, (b * zm - a * zd) / zz
    gm = g * pm.scatter_add_(1, y, torch.full_like(top, -1.0))
    gd = g * pd
    dxm = gm @ wm + gd @ wd
    dxd = gd @ wm + gm @ wd
    dw = (gm.T @ xd + gd.T @ xm) / EPS
    return loss, (dxm.to(dt), dxd.to(dt)), dw.to(dt)


# ---- work and the definition in 64 bits --------------------------------------------
def work(case):
    c = case
    V, d, ob = c["V"], c["d"], 2 if c["dtype"] == "bf16" else 4
    if c["op"].startswith("embed"):
        T, S = c["B"] * c["S"], c["S"] if c["pos"] else 0
        if c["op"] == "embed_fwd":
            rows = min(T, V)
            return {"bytes": 4 * T + (rows + S) * d * (ob + 4) + 8 * T * d, "flops": (4 if c["pos"] else 2) * T * d}
        return {"bytes": 4 * T + 4 * T * d + 4 * (V + S) * d, "flops": T * d}
    T = c["T"]
    by, fl = 2 * ob * (T + V) * d + 12 * T, 6.0 * T * V * d
    if c["op"] == "head_grad":
        by += 2 * ob * T * d + ob * V * d
        fl += 10.0 * T * V * d
    return {"bytes": by, "flops": fl}


def exact(case, seed):
    c = case
    st = _inputs(c, seed)
    f64 = torch.float64
    if c["op"] == "embed_fwd":
        at = []
        for sign in (1.0, -1.0):
            e, v = st["table"]
            x = torch.nn.functional.embedding(st["tok"].long(), e.to(f64) + (sign * EPS) * v.to(f64)) * c["scale"]
            if c["pos"]:
                p, vp = st["table_pos"]
                x = x + (p.to(f64) + (sign * EPS) * vp.to(f64))
            at.append(x.reshape(-1, c["d"]))
        return 0.5 * (at[0] + at[1]), 0.5 * (at[0] - at[1])
    if c["op"] == "embed_bwd":
        # rows in the order of their tokens, then differences of running sums at the tokens' borders
        tok, order = st["tok"].flatten().sort(stable=True)
        run_ = torch.cat([torch.zeros((1, c["d"]), device="cuda", dtype=f64), st["dx"].to(f64)[order].cumsum(0)])
        ids = torch.arange(c["V"], device="cuda", dtype=torch.int32)
        hi = torch.searchsorted(tok.contiguous(), ids, right=True)
        lo = torch.searchsorted(tok.contiguous(), ids)
        e = (run_[hi] - run_[lo]) * c["scale"] / EPS
        if not c["pos"]:
            return e
        p = torch.zeros((c["S"], c["d"]), device="cuda", dtype=f64)
        for b in range(c["B"]):
            p += st["dx"].to(f64)[b * c["S"]:(b + 1) * c["S"]]
        return e, p / EPS
    keep = st["tgt"] >= 0
    res = []
    for sign in (1.0, -1.0):
        x = st["x"][0].to(f64) + sign * st["x"][1].to(f64)
        w = st["w"][0].to(f64) + sign * st["w"][1].to(f64)
        loss, gx, gw = [], [], torch.zeros_like(w)
        for i in range(0, c["T"], 2048):       # rows in turn: a few logits at a time
            r = slice(i, i + 2048)
            p = torch.log_softmax(x[r] @ w.t(), -1)
            k = keep[r].nonzero()[:, 0]
            y = st["tgt"][r][k].long()
            l = torch.zeros(p.shape[0], device="cuda", dtype=f64)
            l[k] = -p[k, y]
            loss.append(l)
            if c["op"] == "head_grad":
                p = p.exp_()
                p[k, y] -= 1.0
                p *= (keep[r].to(f64) * st["scale"])[:, None]
                gx.append(p @ w)
                gw += p.t() @ x[r]
            del p
        res.append((torch.cat(loss), torch.cat(gx) if gx else None, gw))
    (lp, xp, wp), (lm, xm, wm) = res
    loss = 0.5 * (lp + lm), 0.5 * (lp - lm)
    if c["op"] == "head_loss":
        return loss
    return loss, (0.5 * (xp + xm), 0.5 * (xp - xm)), (wp - wm) / (2.0 * EPS)
