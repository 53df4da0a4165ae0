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
