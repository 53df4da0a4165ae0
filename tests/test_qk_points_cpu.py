"""The bounds for heads one of whose points is nearly zero, without a GPU: they let the
norm formed at each point through, and catch the pair's own formula, which loses such
heads, and a result of zeros."""
import pytest

torch = pytest.importorskip("torch")

from tests import qk_ref as R  # noqa: E402

F32, F64 = torch.float32, torch.float64
HQ, HK, DH, T, EPS = 2, 1, 64, 6, 1e-3


def _norm(x, gains, form):
    """Forward without rotation in float32 (sums in float64), the two channels."""
    m, d = (t.view(T, HQ + 2 * HK, DH)[:, :HQ + HK] for t in x)
    q, k, vq, vk = gains
    gm, gd = (torch.cat([a.expand(HQ, DH), b.expand(HK, DH)]).float() for a, b in ((q, k), (EPS * vq, EPS * vk)))
    mean = lambda t: t.mean(-1, keepdim=True)
    M, D = m.double(), d.double()
    if form == "points":
        r = [((mean((M + s * D) ** 2) + 1e-5).rsqrt()).float() for s in (1, -1)]
        z = [((m + s * d) * r[i]) * (gm + s * gd) for i, s in enumerate((1, -1))]
        return 0.5 * (z[0] + z[1]), 0.5 * (z[0] - z[1])
    a, b = mean(M * M + D * D), 2 * mean(M * D)
    rp, rn = ((a + s * b).clamp_min(0) + 1e-5 for s in (1, -1))
    rp, rn = rp.rsqrt(), rn.rsqrt()
    rm, rho = (0.5 * (rp + rn)).float(), (-2 * b * (rp * rn / (rp + rn)) ** 2).float()
    um, ud = (m + d * rho) * rm, (m * rho + d) * rm
    return um * gm + ud * gd, um * gd + ud * gm


@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("size", [1e2, 1e3, 1e5, 1e15, 1e30])
@pytest.mark.parametrize("rest", [0.0, 1e-6])
def test_bounds_of_heads_with_a_small_point(size, sign, rest):
    g = torch.Generator().manual_seed(1)
    rnd = lambda *s: torch.randn(*s, generator=g)
    m = rnd(T, (HQ + 2 * HK) * DH) * size
    x = m, (sign * (1.0 - rest) * m.double()).float()
    gains = 1 + 0.2 * rnd(DH), 1 + 0.2 * rnd(DH), rnd(DH), rnd(DH)
    ang = torch.zeros(T, 1, DH // 2, dtype=F64)
    n = (HQ + HK) * DH
    want = [t[:, :n] for t in R.forward(x, HQ, HK, DH, ang, gains, EPS)]
    bound = R.forward_point_bound(x, HQ, HK, DH, ang, gains, EPS)
    assert float(R.point_ratio(x, HQ, HK, DH).max()) < 2.0 ** -6
    # it is a small fraction of the larger channel everywhere
    assert float((bound / (want[0].abs() + want[1].abs() + 1e-3)).max()) < 1e-4
    for w, y in zip(want, _norm(x, gains, "points")):
        R.check(y.reshape(T, n), w, bound, "points")
    for y in (_norm(x, gains, "pair"), (torch.zeros(T, HQ + HK, DH),) * 2):
        with pytest.raises(AssertionError, match="elements off"):
            for w, t in zip(want, y):
                R.check(t.reshape(T, n), w, bound, "lost")
