"""The work between a decoder layer's q/k/v projection and its attention, timed alone.

Two operators, each forward and backward, in the form in which the library
carries every activation: a pair of tensors, the mean m and the half difference
d over the two points theta +- eps v.

* norm: RMSNorm of every query and key head over its own elements, with a gain
  vector for the queries and one for the keys (parameters, so they have a
  direction and a gradient), and the position rotation in the same pass;
* axes: the rotation alone, where pair i of a head (elements i and i + dh/2)
  turns by the token's position along the axis that pair i belongs to (time,
  height, width).

The value heads behind the keys go through unchanged (forward) or are rounded
to the operand type (backward), so that each call takes a whole projection
output, or its gradient, and gives a whole one.

``run`` without ``own`` is the plain form: products of pairs,
(a b).m = a.m b.m + a.d b.d and (a b).d = a.m b.d + a.d b.m, in elementary
torch operations in float32, angles and the sum over all tokens in float64.
``exact`` evaluates the operators at the two points in float64 instead and
takes the mean and the half difference of the results.
"""
import math

import torch

own = False

EPS = 1e-3
NORM_EPS = 1e-5

# Head counts and widths of the workloads (1.3B: 16 heads of 128; 8B: 32 query
# heads on 8 key/value heads of 128) or generic.
H1B = dict(hq=16, hk=16, dh=128, base=10000.0, dtype="bf16")
H8B = dict(hq=32, hk=8, dh=128, base=500000.0, dtype="bf16")


def listed():
    return [
        # one token of the 1.3B shape: launch latency
        dict(H1B, name="norm fwd one token", op="fwd", norm=True, sections="", inter=False, B=1, S=1, far=0, pad=0),
        # the 1.3B workload's batch, one layer
        dict(H1B, name="norm fwd 1.3B", op="fwd", norm=True, sections="", inter=False, B=4, S=2048, far=0, pad=0),
        # fp32, odd lengths, grouped heads of an uneven width, rows inside a wider buffer
        dict(name="norm fwd odd fp32", op="fwd", norm=True, sections="", inter=False, B=3, S=431, far=0, pad=24,
             hq=6, hk=2, dh=80, base=10000.0, dtype="f32"),
        # an fp32 model's layer with 64-wide heads and interleaved axes, everything in one pass
        dict(name="norm+axes fwd fp32", op="fwd", norm=True, sections="12,10,10", inter=True, B=8, S=1024, far=1000, pad=0,
             hq=16, hk=8, dh=64, base=10000.0, dtype="f32"),
        # the tiny workload's batch: 512 short rows, backward latency
        dict(name="norm bwd tiny fp32", op="bwd", norm=True, sections="", inter=False, B=8, S=64, far=0, pad=0,
             hq=4, hk=4, dh=16, base=10000.0, dtype="f32"),
        # the 1.3B workload's layer, backward with the gains' gradients
        dict(H1B, name="norm bwd 1.3B", op="bwd", norm=True, sections="", inter=False, B=4, S=2048, far=0, pad=0),
        # grouped heads with both: norm and three axes, backward
        dict(H8B, name="norm+axes bwd 8B", op="bwd", norm=True, sections="24,20,20", inter=False, B=1, S=2048, far=100000,
             pad=0),
        # rotation alone: one token far into a video
        dict(H8B, name="axes fwd one token", op="fwd", norm=False, sections="24,20,20", inter=False, B=1, S=1, far=1000000,
             pad=0),
        # the largest: every token that a batch may hold, far positions
        dict(H8B, name="axes fwd 16384 tokens", op="fwd", norm=False, sections="24,20,20", inter=False, B=8, S=2048,
             far=1000000, pad=0),
        # fp32, interleaved axes, 96-wide heads
        dict(name="axes fwd odd fp32", op="fwd", norm=False, sections="16,16,16", inter=True, B=1, S=777, far=5000, pad=8,
             hq=12, hk=4, dh=96, base=10000.0, dtype="f32"),
        # the 8B workload's layer, backward
        dict(H8B, name="axes bwd 8B", op="bwd", norm=False, sections="24,20,20", inter=False, B=1, S=2048, far=100000, pad=0),
        # images: two axes, 72-wide heads, odd lengths
        dict(name="axes bwd odd bf16", op="bwd", norm=False, sections="18,18", inter=False, B=5, S=333, far=300, pad=16,
             hq=9, hk=3, dh=72, base=10000.0, dtype="bf16"),
    ]


def draw(rng):
    dtype = rng.choice(["bf16", "bf16", "f32"])
    dh = rng.choice([128, 128, 64, 8 * rng.randint(1, 32)])
    hk = rng.choice([1, 2, 3, 4, 8, 16])
    hq = hk * rng.choice([1, 1, 2, 3, 4, 8])
    norm = rng.random() < 0.5
    half = dh // 2
    n = 1 if norm and rng.random() < 0.5 else rng.choice([2, 3, 3, 4])
    inter = False
    if n == 1:
        sections = ""
    else:
        inter = rng.random() < 0.5
        if inter:
            rest = [rng.randint(0, half // n) for _ in range(n - 1)]
        else:
            cuts = sorted(rng.randint(0, half) for _ in range(n - 1))
            rest = [b - a for a, b in zip(cuts, cuts[1:] + [half])]
        sections = ",".join(str(s) for s in [half - sum(rest)] + rest)
    case = dict(op=rng.choice(["fwd", "bwd"]), norm=norm, sections=sections, inter=inter, hq=hq, hk=hk, dh=dh,
                base=rng.choice([10000.0, 500000.0]), dtype=dtype, far=rng.choice([0, 1000, 1000000]) if n > 1 else 0,
                pad=8 * rng.choice([0, 0, rng.randint(1, 16)]))
    tokens = int(round(2.0 ** rng.uniform(0.0, 14.0)))
    case["B"] = rng.randint(1, min(8, tokens))
    case["S"] = max(1, tokens // case["B"])
    cap = 7.3e8          # bytes: just below the largest listed cases of each direction
    while work(case)["bytes"] > cap and case["S"] > 1:
        case["S"] = (case["S"] + 1) // 2
    return case


def _sections(c):
    return [int(s) for s in c["sections"].split(",")] if c["sections"] else [c["dh"] // 2]


def _axis_of_pair(c):
    """The axis of each rotated pair: the sections one after the other or, interleaved over n axes,
    pairs a, a + n, ... for axis a >= 1 (as many as its section) and every other pair for axis 0."""
    sec = _sections(c)
    if not c["inter"]:
        return [a for a, s in enumerate(sec) for _ in range(s)]
    out = [0] * sum(sec)
    for a in range(1, len(sec)):
        for j in range(sec[a]):
            out[a + len(sec) * j] = a
    return out


def _dt(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _inputs(c, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    T, dh, dt = c["B"] * c["S"], c["dh"], _dt(c)
    ncol = (c["hq"] + 2 * c["hk"]) * dh

    def rows(dtype, scale_m, scale_d):
        # columns of unequal scale, as a projection gives them; the half difference about EPS below
        col = torch.exp(0.5 * torch.randn(ncol, device="cuda", generator=g))
        out = []
        for s in (scale_m, scale_d):
            full = torch.zeros((T, ncol + c["pad"]), device="cuda", dtype=dtype)
            full[:, :ncol] = (torch.randn((T, ncol), device="cuda", generator=g) * (s * col)).to(dtype)
            out.append(full[:, :ncol])
        return tuple(out)

    st = dict(case=c, x=None, dy=None, gains=None, pos=None)
    if c["norm"] or c["op"] == "fwd":
        st["x"] = rows(dt, 1.0, EPS)
    if c["op"] == "bwd":
        st["dy"] = rows(torch.float32, 1e-4, 1e-4 * EPS)
    if c["norm"]:
        st["gains"] = tuple((1.0 + 0.2 * torch.randn(dh, device="cuda", generator=g)).to(dt) for _ in range(2)) + tuple(
            torch.randn(dh, device="cuda", generator=g) for _ in range(2))
    if c["sections"]:
        # frames of h x w patches in row order, every row of the batch from a start of its own
        B, S, n = c["B"], c["S"], len(_sections(c))
        w = max(1, int(math.sqrt(S) / 2))
        i = torch.arange(S, device="cuda")
        axes = [i // (w * w), i // w % w, i % w, i][:n]
        start = torch.randint(0, c["far"] + 1, (B, 1), device="cuda", generator=g)
        st["pos"] = torch.stack([(start + a).reshape(-1) for a in axes]).to(torch.int32).contiguous()
    return st


def prepare(case, seed):
    st = _inputs(case, seed)
    if own:
        from paper_2602_00816_amd import fdhvp as fd

        c = case
        m = fd.Model("llama", 0, c["hq"] * c["dh"], c["hq"], c["hk"], 8, 8, max(2, c["S"]), c["dtype"], norm_eps=NORM_EPS,
                     rope_base=c["base"], qk_norm=c["norm"], rope_sections=_sections(c) if c["sections"] else None,
                     rope_interleaved=c["inter"])
        T, ncol = c["B"] * c["S"], (c["hq"] + 2 * c["hk"]) * c["dh"]
        st["model"] = m
        st["out"] = tuple(torch.empty((T, ncol), device="cuda", dtype=_dt(c)) for _ in range(2))
        if c["op"] == "bwd" and c["norm"]:
            st["gain_grads"] = tuple(torch.empty(c["dh"], device="cuda") for _ in range(2))
            st["scratch"] = m.qk_scratch(c["B"], c["S"])
    return st


def run(state):
    c = state["case"]
    if own:
        m = state["model"]
        gains = state["gains"]
        if c["op"] == "fwd":
            return m.qk_forward(state["x"], c["S"], gains=gains, eps=EPS, positions=state["pos"], out=state["out"])
        if not c["norm"]:
            return m.qk_backward(state["dy"], c["S"], positions=state["pos"], out=state["out"])
        return m.qk_backward(state["dy"], c["S"], x=state["x"], gains=gains, eps=EPS, positions=state["pos"],
                             out=state["out"], gain_grads=state["gain_grads"], scratch=state["scratch"])
    return _plain_forward(state) if c["op"] == "fwd" else _plain_backward(state)


# ---- the plain form ---------------------------------------------------------------
def _angles(state):
    c = state["case"]
    half = c["dh"] // 2
    inv = c["base"] ** (torch.arange(half, device="cuda", dtype=torch.float64) * (-2.0 / c["dh"]))
    if state["pos"] is None:
        ang = (torch.arange(c["S"], device="cuda", dtype=torch.float64)[:, None] * inv).repeat(c["B"], 1)
    else:
        axis = torch.tensor(_axis_of_pair(c), device="cuda")
        ang = state["pos"].double()[axis].T * inv
    return torch.cos(ang).float()[:, None], torch.sin(ang).float()[:, None]     # [T, 1, half]


def _turn(x, cos, sin):
    h = x.shape[-1] // 2
    a, b = x[..., :h], x[..., h:]
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)


def _mul(a, b):
    return a[0] * b[0] + a[1] * b[1], a[0] * b[1] + a[1] * b[0]


def _gain(state, k):
    g = state["gains"]
    return g[k].float(), EPS * g[2 + k]


def _rms_pair(m, d):
    """Reciprocal root mean squares of m + d and m - d, as a pair."""
    rp = 1.0 / torch.sqrt(((m + d) ** 2).mean(-1, keepdim=True) + NORM_EPS)
    rm = 1.0 / torch.sqrt(((m - d) ** 2).mean(-1, keepdim=True) + NORM_EPS)
    b = 2.0 * (m * d).mean(-1, keepdim=True)
    return 0.5 * (rp + rm), -b * (rp * rm) ** 2 / (rp + rm)


def _heads(c, t):
    x = t.reshape(t.shape[0], -1, c["dh"])
    return x[:, :c["hq"]], x[:, c["hq"]:c["hq"] + c["hk"]], x[:, c["hq"] + c["hk"]:]


def _plain_forward(state):
    c = state["case"]
    cos, sin = _angles(state)
    xm, xd = (_heads(c, t) for t in state["x"])
    ym, yd = [], []
    for k in range(2):
        m, d = xm[k].float(), xd[k].float()
        if c["norm"]:
            m, d = _mul(_mul((m, d), _rms_pair(m, d)), _gain(state, k))
        ym.append(_turn(m, cos, sin).to(_dt(c)))
        yd.append(_turn(d, cos, sin).to(_dt(c)))
    return tuple(torch.cat(y + [x[2]], 1).flatten(1) for y, x in ((ym, xm), (yd, xd)))


def _plain_backward(state):
    c = state["case"]
    cos, sin = _angles(state)
    gm, gd = (_heads(c, t) for t in state["dy"])
    x = [_heads(c, t) for t in state["x"]] if c["norm"] else None
    om, od, dg = [], [], []
    for k in range(2):
        m, d = _turn(gm[k], cos, -sin), _turn(gd[k], cos, -sin)
        if c["norm"]:
            xm, xd = x[0][k].float(), x[1][k].float()
            r = _rms_pair(xm, xd)
            u = _mul((xm, xd), r)
            dg.append(((m * u[1] + d * u[0]).sum((0, 1), dtype=torch.float64) / EPS).float())
            du = _mul((m, d), _gain(state, k))
            ud = _mul(u, du)
            uc = _mul(u, (ud[0].mean(-1, keepdim=True), ud[1].mean(-1, keepdim=True)))
            m, d = _mul(r, (du[0] - uc[0], du[1] - uc[1]))
        om.append(m.to(_dt(c)))
        od.append(d.to(_dt(c)))
    out = tuple(torch.cat(o + [g[2].to(_dt(c))], 1).flatten(1) for o, g in ((om, gm), (od, gd)))
    return (out, tuple(dg)) if c["norm"] else out


# ---- work and the definition in 64 bits --------------------------------------------
def work(case):
    c = case
    T, ob = c["B"] * c["S"], 2 if c["dtype"] == "bf16" else 4
    qk, v = (c["hq"] + c["hk"]) * c["dh"], c["hk"] * c["dh"]
    nax = len(_sections(c)) if c["sections"] else 0
    by = 4 * nax * T + 2 * T * (qk + v) * ob                  # positions; the pair written
    if c["op"] == "fwd":
        by += 2 * T * (qk + v) * ob
        fl = T * qk * (22 if c["norm"] else 6)
    else:
        by += 2 * T * (qk + v) * 4
        if c["norm"]:
            by += 2 * T * qk * ob
        fl = T * qk * (46 if c["norm"] else 6)
    if c["norm"]:
        by += 2 * c["dh"] * (ob + 4 + (4 if c["op"] == "bwd" else 0))
    return {"bytes": by, "flops": fl}


def exact(case, seed):
    c = case
    st = _inputs(c, seed)
    f64 = torch.float64
    T, hq, hk, dh = c["B"] * c["S"], c["hq"], c["hk"], c["dh"]
    if st["pos"] is None:
        pos = torch.arange(c["S"], device="cuda").repeat(c["B"])[:, None].expand(T, dh // 2)
    else:
        pos = torch.stack([st["pos"][a] for a in _axis_of_pair(c)], 1)
    freq = torch.tensor([math.pow(c["base"], -2.0 * i / dh) for i in range(dh // 2)], device="cuda", dtype=f64)
    turn = torch.polar(torch.ones(1, device="cuda", dtype=f64), pos.to(f64) * freq).view(T, 1, dh // 2)
    points = ((1.0, 0), (-1.0, 1))

    def at(pair, sign):
        return (pair[0].to(f64) + sign * pair[1].to(f64)).reshape(T, -1, dh)

    def rotate(x, w):
        z = torch.complex(x[..., :dh // 2].contiguous(), x[..., dh // 2:].contiguous()) * w
        return torch.cat([z.real, z.imag], -1)

    def gains(sign):
        q, k, vq, vk = (t.to(f64) for t in st["gains"])
        return torch.cat([(q + sign * EPS * vq).expand(hq, dh), (k + sign * EPS * vk).expand(hk, dh)])

    res, dgain = [], []
    for sign, _ in points:
        src = at(st["x"] if c["op"] == "fwd" else st["dy"], sign)
        h, v = src[:, :hq + hk], src[:, hq + hk:]
        if c["norm"]:
            x = at(st["x"], sign)[:, :hq + hk]
            s = (x.square().mean(-1, keepdim=True) + NORM_EPS).sqrt()
        if c["op"] == "fwd":
            h = rotate(x / s * gains(sign) if c["norm"] else h, turn)
        else:
            h = rotate(h, turn.conj())
            if c["norm"]:
                dgain.append(tuple(t.sum((0, 1)) for t in (h * x / s).split([hq, hk], 1)))
                a = h * gains(sign)
                h = a / s - x * (a * x).mean(-1, keepdim=True) / s ** 3
        res.append(torch.cat([h, v], 1).flatten(1))
    out = 0.5 * (res[0] + res[1]), 0.5 * (res[0] - res[1])
    if not dgain:
        return out
    return out, tuple((p - q) / (2.0 * EPS) for p, q in zip(*dgain))
