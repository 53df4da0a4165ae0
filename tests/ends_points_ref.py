"""Inputs of the vocabulary loss whose two points are apart in x and in w alike, and what the
kernels' arithmetic may add to its float64 statement there: every product of the pair counts, none is
allowed to be missing."""
import torch

from tests import ends_ref as R

F64 = torch.float64
U = 2.0 ** -24      # half a step of fp32


def inputs(T, V, d, dtype, reach, seed, ignore=0.1):
    """x, w (pairs on the CPU) and targets: half differences of x and w in the same proportion to
    their means, the largest of the logits' near reach."""
    g = torch.Generator().manual_seed(seed)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    xm, xd = (torch.randn(T, d, generator=g) for _ in range(2))
    wm, wd = (torch.randn(V, d, generator=g) * (2.0 / d ** 0.5) for _ in range(2))
    f = reach / float((xd @ wm.T + xm @ wd.T).abs().max())
    x, w = (xm.to(dt), (f * xd).to(dt)), (wm.to(dt), (f * wd).to(dt))
    tgt = torch.randint(0, V, (T,), generator=g)
    tgt[torch.rand(T, generator=g) < ignore] = R.IGNORE
    return x, w, tgt.to(torch.int32)


def statement(x, w, tgt, scale, eps, xdwd=True, gdwd=True):
    """Loss, dx and dw in the pair form; without xdwd or gdwd the product of two half differences is
    left out of the logits' mean or of dx's."""
    live = (tgt.long() != R.IGNORE)[:, None].to(F64)
    (xm, xd), (wm, wd) = (tuple(R.f64(a) for a in p) for p in (x, w))
    lm, ld = xm @ wm.T, xd @ wm.T + xm @ wd.T
    if xdwd:
        lm = lm + xd @ wd.T
    y = tgt.long().clamp(min=0)
    rows = torch.arange(len(y))
    loss, g = [], []
    for l in (lm + ld, lm - ld):
        lp = torch.log_softmax(l, -1)
        loss.append(-lp[rows, y] * live[:, 0])
        p = lp.exp()
        p[rows, y] -= 1.0
        g.append(p * live * scale)
    gm, gd = (g[0] + g[1]) / 2, (g[0] - g[1]) / 2
    dxm = gm @ wm + (gd @ wd if gdwd else 0.0)
    return (((loss[0] + loss[1]) / 2, (loss[0] - loss[1]) / 2), (dxm, gd @ wm + gm @ wd), (gm.T @ xd + gd.T @ xm) / eps)


def bound(x, w, tgt, scale, eps):
    """Element by element, beside the rounding of the outputs.

    A sum of n products in fp32: n u of the absolute sum, and as much again for the products of
    split fp32 operands (2^-23 each).  A logit at either point is off by e, the sum of its channels'
    errors.  An exponential e^(lm - c +- ld), c the largest mean and the largest half difference of the
    row: four roundings of an argument of at most (c - lm) + |ld|, and itself 4 u; where it is held as
    cosh and sinh (|ld| < 1/2) an error of one counts up to e^(1/2) < 1.7 in the other, and up to
    e < 3 in a sum of both.  Sums of 128 of them in fp32, 128 u, likewise (512 u).  bf16 models hold the
    exponentials in fp32, which ends at 2^-126: relative to the sum Z = e^(lse - c) of a point, an absolute
    2^-126 e^(c - lse) of every probability (c - lse is at most twice the largest half difference: 1e-12 at 30).
    The logits' gradient is rounded to the operand type.  Products with it: n roundings of the absolute sum."""
    dt = x[0].dtype
    h = max(R.half_step(dt), 2 * U)
    live = (tgt.long() != R.IGNORE)[:, None].to(F64)
    (xm, xd), (wm, wd) = (tuple(R.f64(a) for a in p) for p in (x, w))
    T, K = xm.shape
    V = wm.shape[0]
    am, ad, bm, bd = xm.abs(), xd.abs(), wm.abs(), wd.abs()
    lm, ld = xm @ wm.T + xd @ wd.T, xd @ wm.T + xm @ wd.T
    e = (4 * K + 8) * U * ((am + ad) @ (bm + bd).T)
    c = lm.amax(1, keepdim=True) + ld.abs().amax(1, keepdim=True)
    ex = 3 * 4 * U * (1 + (c - lm) + ld.abs())
    y = tgt.long().clamp(min=0)
    rows = torch.arange(T)
    loss, eg, g = 0.0, 0.0, []
    for l in (lm + ld, lm - ld):
        p = torch.softmax(l, -1)
        end = 2.0 ** -126 * torch.exp(c - torch.logsumexp(l, -1, keepdim=True)) if dt is torch.bfloat16 else 0.0
        z = 512 * U + (p * (ex + e)).sum(1, keepdim=True) + V * end
        loss = loss + 0.5 * (z[:, 0] + e[rows, y])
        eg = eg + p * (ex + e + z + 8 * U) + end
        p[rows, y] -= 1.0
        g.append(p)
    gm, gd = ((g[0] + g[1]) / 2).abs(), ((g[0] - g[1]) / 2).abs()
    s = abs(scale) * live
    em, ed = s * (eg + h * (gm + eg)), s * (eg + h * (gd + eg))
    gm, gd = s * gm, s * gd
    one = 1 + 1e-6
    tiny = torch.finfo(dt).tiny * V
    n = (2 * V + 8) * U
    dxm = em @ bm + ed @ bd + n * (gm @ bm + gd @ bd)
    dxd = ed @ bm + em @ bd + n * (gd @ bm + gm @ bd)
    dw = (em.T @ ad + ed.T @ am + (2 * T + 24) * U * (gm.T @ ad + gd.T @ am)) / eps
    loss = loss * live[:, 0] * one
    return (loss, loss), (dxm * one + tiny, dxd * one + tiny), dw * one + tiny / eps


def whole_limit(x, w):
    """Of the norm of a float32 gradient's error relative to its own: the rounding of the logits' gradient,
    half a step (root of the mean square below 0.6 of that), and the logits', sqrt(2 K) u of the largest
    in each channel, with their exponentials' 4 u of an argument of up to three times the largest."""
    K = x[0].shape[1]
    (xm, xd), (wm, wd) = (tuple(R.f64(a) for a in p) for p in (x, w))
    big = float(((xm @ wm.T + xd @ wd.T).abs() + (xd @ wm.T + xm @ wd.T).abs()).max())
    return R.half_step(x[0].dtype) + 1e-5 + 2 * (2 * K) ** 0.5 * U * big + 4 * U * (1 + 3 * big)


def check(got, x, w, tgt, scale, eps, what):
    """(loss, dx or None, dw or None), gradients in float32, against the two points themselves."""
    loss, dx, dw = got
    wl, wx, ww = R.head(x, w, tgt, scale, eps)
    bl, bx, bw = bound(x, w, tgt, scale, eps)
    for a, v, b, c in zip(loss, wl, bl, "md"):
        R.check(a, v, b, f"{what} loss.{c}")
    if dx is None:
        return
    lim = whole_limit(x, w)
    for a, v, b, c in ((dx[0], wx[0], bx[0], "dx.m"), (dx[1], wx[1], bx[1], "dx.d"), (dw, ww, bw, "dw")):
        n = float(torch.linalg.norm(v))
        r = float(torch.linalg.norm(R.f64(a) - v)) / n
        assert r <= lim, f"{what} {c}: relative error {r:.2e} of the whole, limit {lim:.2e}"
        R.check(a, v, b, f"{what} {c}")
