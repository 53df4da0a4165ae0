"""Float64 statements of the two ends of a model (fdh_embed_*), on the CPU, with the
error that one rounding to the output's type and the kernels' arithmetic may add."""
import torch

F64 = torch.float64


def f64(t):
    return t.detach().cpu().to(F64)


def half_step(t):
    """Half a step of a type, relative to the value."""
    return torch.finfo(t).eps / 2


def check(got, want, bound, what):
    """Every element within half a step of its type plus bound; NaN exactly where want is NaN."""
    g = f64(got)
    assert g.shape == want.shape, (what, g.shape, want.shape)
    nan = torch.isnan(want)
    assert torch.equal(torch.isnan(g), nan), f"{what}: NaN in other places"
    w = torch.where(nan, torch.zeros_like(want), want)
    g = torch.where(nan, torch.zeros_like(g), g)
    tiny = torch.finfo(got.dtype).tiny      # (a result below the type's range may be flushed)
    off = (g - w).abs() - half_step(got.dtype) * w.abs() * (1 + 1e-9) - bound - tiny
    worst = float(off.max()) if off.numel() else 0.0
    assert worst <= 0.0, f"{what}: {int((off > 0).sum())} of {off.numel()} elements off, worst by {worst:.3e} more than allowed"


# ---- embedding ----------------------------------------------------------------------
def embed_forward(tok, table, eps, scale, positions=None):
    """((m, d), (bound m, bound d)): fp64 arithmetic on exact inputs, so the bounds are a few
    steps of fp64."""
    e, ve = table
    B, S = tok.shape
    V = e.shape[0]
    t = tok.cpu().long()
    bad = ((t < 0) | (t >= V)).reshape(-1)
    t = t.clamp(0, V - 1).reshape(-1)
    m = scale * f64(e)[t]
    d = scale * f64(ve)[t] if ve is not None else torch.zeros_like(m)
    am, ad = m.abs(), d.abs()
    if positions is not None:
        p, vp = positions
        r = torch.arange(S).repeat(B)
        m, am = m + f64(p)[r], am + f64(p)[r].abs()
        if vp is not None:
            d, ad = d + f64(vp)[r], ad + f64(vp)[r].abs()
    d, ad = eps * d, eps * ad
    m[bad] = d[bad] = float("nan")
    return (m, d), (am * 2.0 ** -51, ad * 2.0 ** -51)


def embed_backward(dx, tok, V, eps, scale, max_seq=None, base=(None, None)):
    """((hv_e, hv_p or None), bounds): sums of n fp64 terms are off by at most n steps of the
    sum of their absolute values."""
    B, S = tok.shape
    x = f64(dx)
    t = tok.cpu().long().reshape(-1)
    ok = (t >= 0) & (t < V)
    out, bound = [], []

    def add(rows, n_rows, mul, b):
        idx, val = rows
        s = torch.zeros((n_rows, x.shape[1]), dtype=F64).index_add_(0, idx, val)
        a = torch.zeros((n_rows, x.shape[1]), dtype=F64).index_add_(0, idx, val.abs())
        n = torch.bincount(idx, minlength=n_rows).to(F64)[:, None]
        e = 2.0 ** -52 * (n + 4) * a * mul
        s = s * mul
        if b is not None:
            s, e = s + f64(b), e + 2.0 ** -52 * f64(b).abs()
        out.append(s)
        bound.append(e)

    add((t[ok], x[ok]), V, scale / eps, base[0])
    if max_seq is not None:
        add((torch.arange(S).repeat(B), x), max_seq, 1.0 / eps, base[1])
    return out, bound


# ---- loss over the vocabulary ---------------------------------------------------------
IGNORE = -100


def head(x, w, tgt, scale, eps):
    """loss (m, d), dx (m, d), dw in float64 from the two points themselves.  A target outside
    the vocabulary makes its row, and dw, NaN; rows without a target take no part."""
    V = w[0].shape[0]
    t = tgt.cpu().long()
    live = t != IGNORE
    bad = live & ((t < 0) | (t >= V))
    xs = [torch.where(live[:, None], f64(a), torch.zeros(1, dtype=F64)) for a in x]
    y = t.clamp(0, V - 1)
    res = []
    for sign in (1.0, -1.0):
        a, b = xs[0] + sign * xs[1], f64(w[0]) + sign * f64(w[1])
        lp = torch.log_softmax(a @ b.T, -1)
        loss = -lp.gather(1, y[:, None])[:, 0] * live
        g = lp.exp()
        g[torch.arange(len(t)), y] -= 1.0
        g = g * (scale * live.to(F64))[:, None]
        g[bad], loss[bad] = float("nan"), float("nan")
        res.append((loss, g @ b, g.T @ a))
    (lp, xp, wp), (lm, xm, wm) = res
    return ((lp + lm) / 2, (lp - lm) / 2), ((xp + xm) / 2, (xp - xm) / 2), (wp - wm) / (2 * eps)


def head_bound(x, w, tgt, scale, eps):
    """What the kernels' arithmetic may add, element by element, in the same layout.

    u = 2^-24 is half a step of fp32.  A sum of n products in fp32 is off by at most n u times the
    sum of the absolute products (the products of bf16 values are exact, those of fp32 one
    rounding, counted as two more terms).  The exponentials of bf16 models are fp32: relative
    error 4 u (1 + |argument|) with the argument's rounding; their sums in fp32 over up to 128
    terms: 128 u.  The logits' gradient is rounded to the operand type (half a step); the
    product of two half differences is left out of the means."""
    dt = x[0].dtype
    u, h = 2.0 ** -24, half_step(dt)
    live = (tgt.cpu().long() != IGNORE)[:, None].to(F64)
    zero = torch.zeros(1, dtype=F64)
    xm, xd = (torch.where(live > 0, f64(a), zero) for a in x)
    wm, wd = (f64(a) for a in w)
    T, K = xm.shape
    V = wm.shape[0]
    y = tgt.cpu().long().clamp(0, V - 1)
    rows = torch.arange(T)
    am, ad, bm, bd = xm.abs(), xd.abs(), wm.abs(), wd.abs()
    lm, ld = xm @ wm.T + xd @ wd.T, xd @ wm.T + xm @ wd.T
    em = (K + 2) * u * (am @ bm.T) + ad @ bd.T
    ed = (2 * K + 2) * u * (ad @ bm.T + am @ bd.T)
    pp = torch.softmax(lm + ld, -1), torch.softmax(lm - ld, -1)
    p = torch.maximum(*pp)
    pm, pd = (pp[0] + pp[1]) / 2, (pp[0] - pp[1]) / 2
    top = (lm + ld.abs()).amax(1, keepdim=True)
    x_err = 4 * u * (1 + (lm - top).abs() + ld.abs())        # of one exponential, relative
    z_err = 128 * u + (p * (x_err + em)).sum(1, keepdim=True)  # of a sum of them, relative
    ez = (p * ed).sum(1, keepdim=True)
    mean_d = (p * ld.abs()).sum(1, keepdim=True)
    loss_m = z_err + em[rows, y][:, None]
    # the half difference of the sums' logarithms: every term's relative error acts on its |ld|
    loss_d = ez + ed[rows, y][:, None] + (128 * u + x_err.amax(1, keepdim=True) + em.amax(1, keepdim=True)) * 2 * (
        mean_d + (p * ld.abs()).sum(1, keepdim=True))
    rel = x_err + em + z_err + 4 * u
    gm, gd = pm.clone(), pd
    gm[rows, y] -= 1.0
    s = scale * live
    e_gm = s.abs() * (p * rel + u * gm.abs()) + s.abs() * h * (gm.abs() + p * rel)
    e_gd0 = p * (ed + ez) + p * (ld.abs() + mean_d) * rel
    e_gd = s.abs() * (e_gd0 + h * (gd.abs() + e_gd0))
    am_g, ad_g = (s * gm).abs(), (s * gd).abs()
    dx_m = e_gm @ bm + (V + 2) * u * (am_g @ bm) + ad_g @ bd
    dx_d = e_gd @ bm + e_gm @ bd + (2 * V + 4) * u * (ad_g @ bm + am_g @ bd)
    n = T + 8
    dw = (e_gm.T @ ad + e_gd.T @ am + (2 * n + 4) * u * (am_g.T @ ad + ad_g.T @ am)) / eps * (1 + 4 * u)
    one = 1 + 1e-6
    tiny = torch.finfo(dt).tiny * V
    return tuple(b[:, 0] * live[:, 0] * one for b in (loss_m, loss_d)), (dx_m * one + tiny, dx_d * one + tiny), dw * one + tiny / eps


def check_head(got, x, w, tgt, scale, eps, what, base=None):
    """(loss, dx, dw) against the statement, element by element, and as a whole: roundings that are
    independent of each other leave at most twice half a step of the operand type."""
    (loss, dx, dw) = got
    wl, wx, ww = head(x, w, tgt, scale, eps)
    bl, bx, bw = head_bound(x, w, tgt, scale, eps)
    for a, v, b, c in zip(loss, wl, bl, "md"):
        check(a, v, b, f"{what} loss.{c}")
    if dx is None:
        return
    for a, v, b, c in zip(dx, wx, bx, "md"):
        check(a, v, b, f"{what} dx.{c}")
    if base is not None:
        ww, bw = ww + f64(base), bw + 2.0 ** -23 * f64(base).abs()
    check(dw, ww, bw, f"{what} dw")
    if bool(torch.isfinite(ww).all()) and base is None:
        # the logits carry K roundings of half a step of their partial sums, independent of each other: an
        # absolute error of about sqrt(K) 2^-24 of the largest, and as much relative to the probabilities
        # (logits of 500 from 64 columns: 2.4e-4)
        big = float((f64(x[0]).nan_to_num(0, 0, 0) @ f64(w[0]).T).abs().max())
        lim = 2 * half_step(x[0].dtype) + 1e-5 + x[0].shape[1] ** 0.5 * 2.0 ** -24 * big
        for a, v, c in ((dx[0], wx[0], "dx.m"), (dx[1], wx[1], "dx.d"), (dw, ww, "dw")):
            n = float(torch.linalg.norm(v))
            r = float(torch.linalg.norm(f64(a) - v)) / n if n else 0.0
            assert r <= lim, f"{what} {c}: relative error {r:.2e} of the whole"
