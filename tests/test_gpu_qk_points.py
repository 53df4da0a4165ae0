"""Heads whose half difference is close to the mean or its negative, so that one of the two
points is nearly or exactly zero, at every magnitude, beside ordinary heads: each held to
what its two points are worth (tests/qk_ref.py), and no head's bits depend on its
neighbours'."""
import pytest

from tests import qk_ref as R
from tests.gpu_util import need_gpu, say
from tests.test_gpu_qk import BASE, EPS, _dt, _gains, _model, _pair

pytestmark = pytest.mark.gpu

# (magnitude, sign, 1 - x.d / x.m); None: an ordinary head
KINDS = [None] + [(a, s, e) for a in (1.0, 1e2, 1e3, 1e5, 1e15, 1e30, 1e35) for s in (1.0, -1.0) for e in (0.0, 1e-6, 2.0 ** -7)]
# about the ratio at which the smaller point's mean square counts as small: (0.1 / 0.9)^2 and (1 / 7)^2
# lie on either side of 2^-6
KINDS += [(1e3, s, e) for s in (1.0, -1.0) for e in (0.2, 0.25, 0.5)] + [None]


def _heads(torch, hq, hk, dh, dtype, seed):
    """[T] tokens whose q and k heads run through KINDS, and the ordinary heads' mask [T, hq + hk]."""
    H = hq + hk
    T = -(-2 * len(KINDS) // H) + 1
    x = _pair(torch, T, (hq + 2 * hk) * dh, dtype, seed)
    m, d = (t.view(T, hq + 2 * hk, dh) for t in x)
    plain = torch.zeros(T, H, dtype=torch.bool)
    for i in range(T * H):
        t, h, kind = i // H, i % H, KINDS[i % len(KINDS)]
        if kind is None:
            plain[t, h] = True
            continue
        a, s, e = kind
        m[t, h] = (m[t, h].float() * a).to(dtype)
        d[t, h] = (s * (1.0 - e) * m[t, h].double()).to(dtype)
    return x, plain


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hk,dh", [(1, 1, 8), (4, 4, 16), (2, 1, 48), (5, 5, 40), (8, 2, 128), (3, 1, 72), (3, 1, 152), (1, 1, 256)])
def test_one_point_nearly_zero(hq, hk, dh, dtype):
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    dt, H = _dt(torch, dtype), hq + hk
    m = _model(fd, hq, hk, dh, dtype)
    x, plain = _heads(torch, hq, hk, dh, dt, 3)
    T, n = x[0].shape[0], H * dh
    gains = _gains(torch, dh, dt, 5)
    ang = R.angles(dh, BASE, T, T)
    near = R.point_ratio(x, hq, hk, dh) < 0.999 * 2.0 ** -6
    cols = near[:, :, None].expand(T, H, dh).reshape(T, n)
    say(f"{hq}/{hk} heads of {dh} {dtype}: {int(near.sum())} of {T * H} heads with a small point")

    def either(point, pair):
        return torch.where(cols, point, pair[:, :n])

    y = m.qk_forward(x, T, gains=gains, eps=EPS)
    want = R.forward(x, hq, hk, dh, ang, gains, EPS)
    pb = R.forward_point_bound(x, hq, hk, dh, ang, gains, EPS)
    for g, w, b, c in zip(y, want, R.forward_bound(x, hq, hk, dh, ang, gains, EPS), "md"):
        R.check(g[:, :n], w[:, :n], either(pb, b), f"y.{c}")
    assert all(torch.equal(a[:, n:], b[:, n:]) for a, b in zip(y, x))

    # a gradient at both points alike, and one that all but leaves a point out
    ncol = (hq + 2 * hk) * dh
    for name, dy in (("even", _pair(torch, T, ncol, torch.float32, 7)),
                     ("one point", (lambda t: (t, t * (1.0 - 1e-6)))(_pair(torch, T, ncol, torch.float32, 8)[0]))):
        dx, dg = m.qk_backward(dy, T, x=x, gains=gains, eps=EPS)
        want, wg = R.backward(x, dy, hq, hk, dh, ang, gains, EPS)
        pb, _ = R.backward_point_bound(x, dy, hq, hk, dh, ang, gains, EPS)
        b, _ = R.backward_bound(x, dy, hq, hk, dh, ang, gains, EPS)
        for g, w, e, c in zip(dx, want, b, "md"):
            R.check(g[:, :n], w[:, :n], either(pb, e), f"{name}: dx.{c}")
        # (the gains' sums are linear in dy: either kind of head with the other's gradient cleared)
        part = [tuple((t.cpu().view(T, hq + 2 * hk, dh)[:, :H] * k[:, :, None]) for t in dy) for k in (near, ~near)]
        part = [tuple(torch.cat([t, torch.zeros(T, hk, dh)], 1).view(T, ncol) for t in p) for p in part]
        pg = R.backward_point_bound(x, part[0], hq, hk, dh, ang, gains, EPS)[1]
        og = R.backward_bound(x, part[1], hq, hk, dh, ang, gains, EPS)[1]
        for g, w, e, f, c in zip(dg, wg, pg, og, "qk"):
            R.check(g, w, e + f, f"{name}: dg.{c}")


@pytest.mark.parametrize("hq,hk,dh,dtype", [(4, 4, 16, "f32"), (8, 2, 128, "bf16"), (5, 5, 40, "f32"), (3, 1, 152, "f32")])
def test_ordinary_heads_keep_their_bits_beside_them(hq, hk, dh, dtype):
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    dt, H = _dt(torch, dtype), hq + hk
    m = _model(fd, hq, hk, dh, dtype)
    x, plain = _heads(torch, hq, hk, dh, dt, 3)
    T = x[0].shape[0]
    other = _pair(torch, T, (hq + 2 * hk) * dh, dt, 4)
    keep = torch.cat([plain, torch.ones(T, hk, dtype=torch.bool)], 1).cuda()[:, :, None].expand(T, H + hk, dh).reshape(T, -1)
    z = tuple(torch.where(keep, a, b) for a, b in zip(x, other))
    gains = _gains(torch, dh, dt, 5)
    dy = _pair(torch, T, (hq + 2 * hk) * dh, torch.float32, 6)
    for a, b in zip((*m.qk_forward(x, T, gains=gains, eps=EPS), *m.qk_backward(dy, T, x=x, gains=gains, eps=EPS)[0]),
                    (*m.qk_forward(z, T, gains=gains, eps=EPS), *m.qk_backward(dy, T, x=z, gains=gains, eps=EPS)[0])):
        assert torch.equal(a[keep], b[keep])
    # in place, and the same call again
    y = m.qk_forward(x, T, gains=gains, eps=EPS)
    w = tuple(t.clone() for t in x)
    m.qk_forward(w, T, gains=gains, eps=EPS, out=w)
    assert all(torch.equal(a, b) for a, b in zip(w, y))


@pytest.mark.parametrize("hq,hk,dh,dtype", [(8, 2, 128, "bf16"), (4, 1, 128, "f32"), (16, 16, 16, "f32"), (3, 1, 152, "bf16")])
def test_a_few_of_them_in_a_long_batch(hq, hk, dh, dtype):
    """Several steps per wavefront, most of them without such a head: the gain gradients,
    and every row's bits as in calls on parts of the batch."""
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    dt, H, T, part = _dt(torch, dtype), hq + hk, 64 * 150 + 7, 64 * 30
    ncol, n = (hq + 2 * hk) * dh, (hq + hk) * dh
    m = _model(fd, hq, hk, dh, dtype)
    x = _pair(torch, T, ncol, dt, 3)
    a, b = (t.view(T, hq + 2 * hk, dh) for t in x)
    g = torch.Generator().manual_seed(5)
    few = (torch.rand(T, H, generator=g) < 0.003).nonzero().cuda()
    few = torch.cat([few, torch.tensor([[0, 0], [T - 1, H - 1]], device="cuda")])
    a[few[:, 0], few[:, 1]] *= 1e5
    b[few[:, 0], few[:, 1]] = -a[few[:, 0], few[:, 1]]
    dy = _pair(torch, T, ncol, torch.float32, 4, scale=(1.0, 0.5))
    gains = _gains(torch, dh, dt, 5)
    pos = torch.randint(0, 1000, (1, T), dtype=torch.int32, device="cuda")
    y = m.qk_forward(x, T, gains=gains, eps=EPS, positions=pos)
    dx, dg = m.qk_backward(dy, T, x=x, gains=gains, eps=EPS, positions=pos)
    for s in range(0, T, part):
        e = min(T, s + part)
        cut = lambda p: tuple(t[s:e] for t in p)
        p = pos[:, s:e].contiguous()
        ys = m.qk_forward(cut(x), e - s, gains=gains, eps=EPS, positions=p)
        ds, _ = m.qk_backward(cut(dy), e - s, x=cut(x), gains=gains, eps=EPS, positions=p)
        for big, small in zip((*y, *dx), (*ys, *ds)):
            assert torch.equal(big[s:e], small), (s, e)
    again = m.qk_backward(dy, T, x=x, gains=gains, eps=EPS, positions=pos)[1]
    assert all(torch.equal(p, q) for p, q in zip(again, dg))
    ang = R.angles(dh, BASE, T, T, pos)
    near = R.point_ratio(x, hq, hk, dh) < 2.0 ** -6
    say(f"{hq}/{hk} heads of {dh} {dtype}: {int(near.sum())} of {T * H} heads with a small point")
    assert int(near.sum()) >= few.unique(dim=0).shape[0]
    _, wg = R.backward(x, dy, hq, hk, dh, ang, gains, EPS)
    mask = torch.cat([near, torch.zeros(T, hk, dtype=torch.bool)], 1)[:, :, None].expand(T, H + hk, dh).reshape(T, ncol)
    cleared = [tuple(t.cpu() * k for t in dy) for k in (mask, ~mask)]
    pg = R.backward_point_bound(x, cleared[0], hq, hk, dh, ang, gains, EPS)[1]
    og = R.backward_bound(x, cleared[1], hq, hk, dh, ang, gains, EPS)[1]
    for p, w, e, f, c in zip(dg, wg, pg, og, "qk"):
        R.check(p, w, e + f, f"dg.{c}")


def test_replayed_in_a_graph():
    """Heads with a small point in some replays, at places that change, and in none."""
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    hq, hk, dh, T = 4, 1, 128, 700
    ncol = (hq + 2 * hk) * dh
    side = torch.cuda.Stream()
    m, eager = _model(fd, hq, hk, dh, "f32", stream=side.cuda_stream), _model(fd, hq, hk, dh, "f32")
    gains = _gains(torch, dh, torch.float32, 1)
    x = _pair(torch, T, ncol, torch.float32, 2)
    dy = _pair(torch, T, ncol, torch.float32, 3)
    y, dx = (tuple(torch.empty_like(t) for t in x) for _ in range(2))
    dg = tuple(torch.empty(dh, device="cuda") for _ in range(2))
    sc = m.qk_scratch(1, T)
    side.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(g, stream=side):
            m.qk_forward(x, T, gains=gains, eps=EPS, out=y)
            m.qk_backward(dy, T, x=x, gains=gains, eps=EPS, out=dx, gain_grads=dg, scratch=sc)
    torch.cuda.synchronize()
    for step, few in enumerate((0, 5, 0, T, 1)):
        for t, s in zip(x, _pair(torch, T, ncol, torch.float32, 10 + step)):
            t.copy_(s)
        rows = torch.randperm(T, generator=torch.Generator().manual_seed(step))[:few].cuda()
        x[0][rows] *= 1e4
        x[1][rows] = x[0][rows] if step % 2 else -x[0][rows]
        want = (*eager.qk_forward(x, T, gains=gains, eps=EPS),)
        wdx, wdg = eager.qk_backward(dy, T, x=x, gains=gains, eps=EPS)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((*y, *dx, *dg), (*want, *wdx, *wdg))), step
