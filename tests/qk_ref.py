"""Plain float64 statement of the q/k front of a layer: per-head RMSNorm and
rotation, written for one point (PyTorch on the CPU, gradients by autograd) and
evaluated at the two points of a pair; and bounds for the error of fp32
arithmetic on pairs, from sums of absolute values."""
import torch

F64 = torch.float64
U32 = 2.0 ** -24                                        # half a step of float32


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def axis_of_pairs(half, sections, interleaved):
    n = len(sections)
    if n < 2:
        return torch.zeros(half, dtype=torch.long)
    if not interleaved:
        return torch.repeat_interleave(torch.arange(n), torch.tensor(sections))
    axis = torch.zeros(half, dtype=torch.long)
    for a in range(1, n):
        for j in range(sections[a]):
            axis[a + n * j] = a
    return axis


def angles(dh, base, T, seq, positions=None, sections=(), interleaved=False):
    """[T, 1, dh/2] angles in float64."""
    half = dh // 2
    inv = torch.tensor([base ** (-2.0 * i / dh) for i in range(half)], dtype=F64)
    if positions is None:
        p = (torch.arange(T) % seq).to(F64)[:, None].expand(T, half)
    else:
        p = positions.cpu().reshape(-1, T).to(F64)[axis_of_pairs(half, sections, interleaved)].T
    return (p * inv)[:, None]


def front(x, hq, hk, dh, ang, gains=None, eps=1e-5):
    """One point: x float64 [T, (hq + 2 hk) dh] -> y; gains (q, k) or None."""
    T = x.shape[0]
    h = x.view(T, hq + 2 * hk, dh)
    q, k, v = h.split([hq, hk, hk], 1)
    if gains is not None:
        q = q / torch.sqrt((q * q).mean(-1, keepdim=True) + eps) * gains[0]
        k = k / torch.sqrt((k * k).mean(-1, keepdim=True) + eps) * gains[1]
    c, s = torch.cos(ang), torch.sin(ang)

    def turn(z):
        a, b = z[..., :dh // 2], z[..., dh // 2:]
        return torch.cat([a * c - b * s, b * c + a * s], -1)

    return torch.cat([turn(q), turn(k), v], 1).reshape(T, -1)


def points(pair):
    m, d = (t.detach().cpu().to(F64) for t in pair)
    return m + d, m - d


def as_pair(p, q):
    return 0.5 * (p + q), 0.5 * (p - q)


def gains_at(gains, eps, sign):
    if gains is None:
        return None
    q, k, vq, vk = (None if g is None else g.detach().cpu().to(F64) for g in gains)
    return tuple(g if v is None else g + sign * eps * v for g, v in ((q, vq), (k, vk)))


def forward(x, hq, hk, dh, ang, gains=None, eps=1.0, norm_eps=1e-5):
    return as_pair(*(front(p, hq, hk, dh, ang, gains_at(gains, eps, s), norm_eps) for p, s in zip(points(x), (1, -1))))


def backward(x, dy, hq, hk, dh, ang, gains=None, eps=1.0, norm_eps=1e-5):
    """(dx pair, (dq, dk) or None): gradients at the two points by autograd."""
    dx, dg = [], []
    for p, w, s in zip(points(x), points(dy), (1, -1)):
        p = p.requires_grad_(True)
        g = gains_at(gains, eps, s)
        leaves = [p]
        if g is not None:
            g = tuple(t.clone().requires_grad_(True) for t in g)
            leaves += list(g)
        out = torch.autograd.grad((front(p, hq, hk, dh, ang, g, norm_eps) * w).sum(), leaves)
        dx.append(out[0])
        dg.append(out[1:])
    dgain = None if gains is None else tuple((a - b) / (2.0 * eps) for a, b in zip(*dg))
    return as_pair(*dx), dgain


# ---- error bounds ------------------------------------------------------------------
# A chain of fp32 operations on non-negative terms is off by at most (number of
# roundings) * 2^-24 of the sum of the terms' absolute values, up to terms of
# 2^-48; the bounds below are those sums, and the factors count, along the longest
# path from the inputs to the output, every operation and every fp32 rounding of a
# precomputed factor (r.m, rho = r.d / r.m, the gain's half difference, cosine and sine).
# The statement itself takes a difference of two points of the size of the mean, each
# formed in float64 by fewer than 32 operations: its half difference is off by up to
# 32 * 2^-53 of the mean channel's sum of absolute values, which every bound includes
# (it counts where the half difference is 2^-24 of the mean or less).
REF = 32 * 2.0 ** -53


def _mul(a, b):
    return a[0] * b[0] + a[1] * b[1], a[0] * b[1] + a[1] * b[0]


def _abs_parts(x, hq, hk, dh, gains, eps, norm_eps):
    T = x[0].shape[0]
    xm, xd = (t.detach().cpu().to(F64).view(T, hq + 2 * hk, dh)[:, :hq + hk] for t in x)
    sp = ((xm + xd) ** 2).mean(-1, keepdim=True) + norm_eps
    sm = ((xm - xd) ** 2).mean(-1, keepdim=True) + norm_eps
    r = as_pair(sp.rsqrt(), sm.rsqrt())
    # (r.d is formed from mean(m d) relative to that sum of signed terms, in fp64)
    r = r[0].abs(), r[1].abs()
    q, k, vq, vk = (torch.zeros(dh, dtype=F64) if t is None else t.detach().cpu().to(F64).abs() for t in gains)
    g = tuple(torch.cat([a.expand(hq, dh), b.expand(hk, dh)]) for a, b in ((q, k), (eps * vq, eps * vk)))
    return (xm.abs(), xd.abs()), r, g


def _abs_turn(z, ang):
    # An angle is a frequency (a power, good to 2^-51 or so, on either side) times a
    # position, one more rounding here: the two sides' angles differ by up to
    # 2^-50 |ang|, cosine and sine by that times the other one.  Counted as
    # 2^-50 / 2^-24 of a rounding.
    c, s = torch.cos(ang).abs(), torch.sin(ang).abs()
    e = 2.0 ** -50 / U32 * ang.abs()
    c, s = c + e * s, s + e * c
    h = z.shape[-1] // 2
    a, b = z[..., :h], z[..., h:]
    return torch.cat([a * c + b * s, b * c + a * s], -1)


def _bounds(z, k, src, hq, hk, dh):
    """Bounds of whole rows: the turned columns from z, the value columns exact."""
    T = src[0].shape[0]
    mean = sum(t.detach().cpu().to(F64).abs() for t in src).view(T, hq + 2 * hk, dh)
    mean = torch.cat([z[0], mean[:, hq + hk:]], 1)
    out = []
    for c in z:
        b = REF * mean
        b[:, :hq + hk] += (k + 1) * U32 * c
        out.append(b.reshape(T, -1))
    return out


def forward_bound(x, hq, hk, dh, ang, gains=None, eps=1.0, norm_eps=1e-5):
    """Bounds (m, d) of the arithmetic's error: norm 8 roundings (rho, x rho, +,
    r.m, times r.m, gain, times gain, +), rotation 3 (cosine, product, +), and one for what the products of
    roundings add."""
    k = 3
    if gains is None:
        z = tuple(t.detach().cpu().to(F64).abs().view(-1, hq + 2 * hk, dh)[:, :hq + hk] for t in x)
    else:
        ax, r, g = _abs_parts(x, hq, hk, dh, gains, eps, norm_eps)
        z = _mul(_mul(ax, r), g)
        k += 8
    return _bounds([_abs_turn(c, ang) for c in z], k, x, hq, hk, dh)


def backward_bound(x, dy, hq, hk, dh, ang, gains=None, eps=1.0, norm_eps=1e-5):
    """Bounds (m, d) for dx and for the two gain gradients.  dz: 3 roundings; du = dz o g: 3
    more; u: 5; u o du: 12 with the product; c, its mean in fp32: 16 sums in a lane, 5 over
    lanes, 1 division: 34; u o c: 5 and 2 more, 41; du - u o c: 42; times r: 5 more, 47.  Gain terms: dz 3, u 5, product and sum 2, the output's own rounding 1."""
    T = dy[0].shape[0]
    z = [_abs_turn(t.detach().cpu().to(F64).abs().view(T, hq + 2 * hk, dh)[:, :hq + hk], ang) for t in dy]
    dg = None
    k = 3
    if gains is not None:
        ax, r, g = _abs_parts(x, hq, hk, dh, gains, eps, norm_eps)
        u = _mul(ax, r)
        t = (11 * U32 * (z[0] * u[1] + z[1] * u[0]) + REF * (z[0] * u[0] + z[1] * u[1])) / eps
        dg = t[:, :hq].sum((0, 1)), t[:, hq:].sum((0, 1))
        du = _mul(z, g)
        ud = _mul(ax, du)
        c = _mul(r, (ud[0].mean(-1, keepdim=True), ud[1].mean(-1, keepdim=True)))
        uc = _mul(u, c)
        z = _mul(r, (du[0] + uc[0], du[1] + uc[1]))
        k = 47
    return _bounds(z, k, dy, hq, hk, dh), dg


def check(got, want, bound, what):
    """|got - want| <= half a step of got's type + bound, element by element."""
    g = got.detach().cpu().to(F64)
    tol = half_step(got.dtype) * (want.abs() + bound) + bound + torch.finfo(got.dtype).tiny
    bad = ~((g - want).abs() <= tol)
    assert not bad.any(), (f"{what}: {int(bad.sum())} of {bad.numel()} elements off, worst "
                           f"{float(((g - want).abs() / tol).nan_to_num(float('inf')).max()):.3g} x the bound")


# ---- heads one of whose points is much smaller than the other -------------------------
# Where x.d is close to x.m or -x.m, the sums above are much larger than the result
# (|x.m| r.m + |x.d| |r.d| against |u+| + |u-|, as r of the small point is the larger),
# so a result that has lost every digit would pass.  Such heads are held to sums of
# absolute values taken at each point on its own, in which nothing cancels; a mean or
# half difference is off by half of what its two points are off by together.
def point_ratio(x, hq, hk, dh, norm_eps=1e-5):
    """[T, hq + hk]: the smaller of a head's mean squares (with epsilon) over the larger."""
    s = [(p.view(-1, hq + 2 * hk, dh)[:, :hq + hk] ** 2).mean(-1) + norm_eps for p in points(x)]
    return torch.minimum(*s) / torch.maximum(*s)


def _point_parts(x, hq, hk, dh, gains, eps, norm_eps):
    """|u| and r at each point, and |gain| + |its half difference|."""
    q, k, vq, vk = (torch.zeros(dh, dtype=F64) if t is None else t.detach().cpu().to(F64).abs() for t in gains)
    g = torch.cat([(q + eps * vq).expand(hq, dh), (k + eps * vk).expand(hk, dh)])
    out = []
    for p in points(x):
        p = p.view(-1, hq + 2 * hk, dh)[:, :hq + hk]
        r = ((p * p).mean(-1, keepdim=True) + norm_eps).rsqrt()
        out.append((p.abs() * r, r))
    return out, g


def forward_point_bound(x, hq, hk, dh, ang, gains, eps=1.0, norm_eps=1e-5):
    """Bound of either channel's turned columns, [T, (hq + hk) dh].  u is formed as
    ((m -+ d) + d kappa) r.m, kappa = 2 r / (r+ + r-) with the smaller r: with |d|, |m| <=
    (|x+| + |x-|) / 2 and one r at least 8 times the other, the terms' sum is at most 5/4 of
    (|u+| + |u-|) / 2.  Roundings: difference (or kappa) and sum 2, r.m and its product 4, gain's half
    difference, product, sum 7; rotation 10; and one for what the products of roundings
    add: 11, of 5/4: 14."""
    parts, g = _point_parts(x, hq, hk, dh, gains, eps, norm_eps)
    b = 0.5 * sum(_abs_turn(u * g, ang) for u, _ in parts)
    return ((14 * U32 + REF) * b).reshape(b.shape[0], -1)


def backward_point_bound(x, dy, hq, hk, dh, ang, gains, eps=1.0, norm_eps=1e-5):
    """(bound of either channel of dx's turned columns, of the two gain gradients).  Roundings: dy.m
    +- dy.d, rotation 3: dz 4; gain 2, product: du 7; u: 3; u du 11; its mean in fp32, 16 sums in
    a lane, 5 over lanes, 1 / n and its product: c 34; u c 38; du - u c 39; r and its product 41; half
    the sum of two points 42; one more as above.  Gain terms: dz 4, u 3, product, difference: 9, and one."""
    parts, g = _point_parts(x, hq, hk, dh, gains, eps, norm_eps)
    z = [_abs_turn(p.abs().view(-1, hq + 2 * hk, dh)[:, :hq + hk], ang) for p in points(dy)]
    b = 0.5 * sum(r * (a * g + u * (u * a * g).mean(-1, keepdim=True)) for (u, r), a in zip(parts, z))
    t = (10 * U32 + REF) * 0.5 * sum(u * a for (u, _), a in zip(parts, z)) / eps
    return ((43 * U32 + REF) * b).reshape(b.shape[0], -1), (t[:, :hq].sum((0, 1)), t[:, hq:].sum((0, 1)))
