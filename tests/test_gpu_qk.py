"""The q/k front of a layer (fdh_qk_forward, fdh_qk_backward) against the float64
statement of tests/qk_ref.py: head counts and widths, types, one token to some
hundred, strides, axes, far positions, gains with and without a direction, values at
the ends of the range, NaN and infinities, in place, accumulation, repeated calls,
graphs, other streams.  Every element is held to half a step of its type plus a
bound of the fp32 arithmetic's error that is worked out beside it in qk_ref."""
import gc

import numpy as np
import pytest

from tests import qk_ref as R
from tests.gpu_util import need_gpu, say

pytestmark = pytest.mark.gpu

BASE = 10000.0
EPS = 1e-3
# (query heads, key heads, head width): each power of two of lanes per head, widths
# that fill them and that do not, heads that fill a wavefront and that do not
HEADS = [(1, 1, 8), (3, 1, 16), (4, 2, 24), (5, 5, 40), (6, 2, 64), (9, 3, 72), (2, 2, 80), (4, 1, 96), (8, 2, 128),
         (3, 3, 152), (2, 1, 248), (1, 1, 256)]


def _model(fd, hq, hk, dh, dtype, norm=True, sections=None, inter=False, **kw):
    return fd.Model("llama", 0, hq * dh, hq, hk, 8, 8, 64, dtype, rope_base=BASE, qk_norm=norm, rope_sections=sections,
                    rope_interleaved=inter, **kw)


def _pair(torch, T, ncol, dtype, seed, pad=0, scale=(1.0, EPS)):
    g = torch.Generator().manual_seed(seed)
    out = []
    for s in scale:
        full = torch.full((T, ncol + pad), 7.0, dtype=dtype)
        full[:, :ncol] = (torch.randn(T, ncol, generator=g) * s).to(dtype)
        out.append(full.cuda()[:, :ncol])
    return tuple(out)


def _gains(torch, dh, dtype, seed, direction=True):
    g = torch.Generator().manual_seed(seed)
    q, k = ((1.0 + 0.2 * torch.randn(dh, generator=g)).to(dtype).cuda() for _ in range(2))
    return (q, k) + (tuple(torch.randn(dh, generator=g).cuda() for _ in range(2)) if direction else (None, None))


def _dt(torch, dtype):
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def _check_forward(torch, m, x, seq, hq, hk, dh, gains, pos, sections=(), inter=False, out=None, what=""):
    y = m.qk_forward(x, seq, gains=gains, eps=EPS, positions=pos, out=out)
    torch.cuda.synchronize()
    ang = R.angles(dh, BASE, x[0].shape[0], seq, pos, sections, inter)
    want = R.forward(x, hq, hk, dh, ang, gains, EPS)
    bound = R.forward_bound(x, hq, hk, dh, ang, gains, EPS)
    for g, w, b, c in zip(y, want, bound, "md"):
        R.check(g, w, b, f"{what} y.{c}")
    v = (hq + hk) * dh
    assert all(torch.equal(a[:, v:], b[:, v:]) for a, b in zip(y, x))
    return y


def _check_backward(torch, m, x, dy, seq, hq, hk, dh, gains, pos, sections=(), inter=False, out=None, what="", **kw):
    got = m.qk_backward(dy, seq, x=x, gains=gains, eps=EPS, positions=pos, out=out, **kw)
    torch.cuda.synchronize()
    dx, dg = got if gains is not None else (got, None)
    ang = R.angles(dh, BASE, dy[0].shape[0], seq, pos, sections, inter)
    want, wg = R.backward(x if x is not None else dy, dy, hq, hk, dh, ang, gains, EPS)
    bound, bg = R.backward_bound(x, dy, hq, hk, dh, ang, gains, EPS)
    for g, w, b, c in zip(dx, want, bound, "md"):
        R.check(g, w, b, f"{what} dx.{c}")
    if gains is not None:
        for g, w, b, c in zip(dg, wg, bg, "qk"):
            R.check(g, w, b, f"{what} dg.{c}")
    return dx, dg


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hk,dh", HEADS)
def test_norm_and_rotation(hq, hk, dh, dtype):
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    dt, ncol = _dt(torch, dtype), (hq + 2 * hk) * dh
    m = _model(fd, hq, hk, dh, dtype)
    for i, (B, S, pad) in enumerate([(1, 1, 0), (1, 2, 8), (3, 7, 24), (2, 65, 0), (1, 257, 8), (70, 1, 0), (43, 3, 8)]):
        x = _pair(torch, B * S, ncol, dt, 10 + i, pad)
        dy = _pair(torch, B * S, ncol, torch.float32, 20 + i, pad, (1e-4, 1e-7))
        gains = _gains(torch, dh, dt, 30 + i, direction=i != 2)
        what = f"{hq}/{hk} heads of {dh}, {B}x{S} {dtype}"
        say(what)
        _check_forward(torch, m, x, S, hq, hk, dh, gains, None, what=what)
        _check_backward(torch, m, x, dy, S, hq, hk, dh, gains, None, what=what)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("hq,hk,dh,sections,inter", [
    (4, 2, 24, (12,), False), (4, 2, 24, (4, 4, 4), False), (4, 2, 24, (6, 4, 2), True), (6, 3, 72, (18, 18), False),
    (5, 1, 40, (0, 0, 20), False), (3, 1, 64, (8, 8, 8, 8), True), (8, 2, 128, (24, 20, 20), True), (2, 1, 256, (100, 27, 1), False)])
def test_axes(hq, hk, dh, sections, inter, norm, dtype):
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    dt, ncol = _dt(torch, dtype), (hq + 2 * hk) * dh
    m = _model(fd, hq, hk, dh, dtype, norm, sections, inter)
    rng = np.random.default_rng(7)
    for i, (B, S, lim) in enumerate([(1, 1, 10 ** 6), (2, 19, 300), (1, 130, 2 ** 24)]):
        T = B * S
        x = _pair(torch, T, ncol, dt, 40 + i, 8 * i)
        dy = _pair(torch, T, ncol, torch.float32, 50 + i, 8 * i, (1.0, EPS))
        gains = _gains(torch, dh, dt, 60 + i) if norm else None
        pos = torch.from_numpy(rng.integers(-lim, lim, (len(sections), B, S)).astype(np.int32)).cuda()
        what = f"{hq}/{hk} heads of {dh}, axes {sections} {'interleaved ' if inter else ''}{B}x{S} {dtype}"
        say(what)
        _check_forward(torch, m, x, S, hq, hk, dh, gains, pos, sections, inter, what=what)
        _check_backward(torch, m, x if norm else None, dy, S, hq, hk, dh, gains, pos, sections, inter, what=what)
        # text: no positions are the positions 0 .. S - 1 on every axis, to the bit
        y0 = m.qk_forward(x, S, gains=gains, eps=EPS)
        ar = torch.arange(S, dtype=torch.int32, device="cuda").repeat(len(sections) * B)
        y1 = m.qk_forward(x, S, gains=gains, eps=EPS, positions=ar)
        assert all(torch.equal(a, b) for a, b in zip(y0, y1))


def test_positions_at_the_ends_of_int32():
    """cos and sin in fp32 are off by half a step; the angle itself carries the
    rounding of the frequency and, in the reference, of its product with the position:
    2^-52 of at most 2^31 radians each, 1e-6 in all."""
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    hq, hk, dh = 2, 1, 16
    m = _model(fd, hq, hk, dh, "f32", False)
    pos = torch.tensor([-2 ** 31, 2 ** 31 - 1, -2 ** 31 + 1, 2 ** 30, -1, 0, 1], dtype=torch.int32, device="cuda")
    T = pos.numel()
    x = _pair(torch, T, (hq + 2 * hk) * dh, torch.float32, 1)
    y = m.qk_forward(x, T, positions=pos)
    want = R.forward(x, hq, hk, dh, R.angles(dh, BASE, T, T, pos))
    for g, w, s in zip(y, want, x):
        lim = (1e-6 + 4 * R.U32) * 2 * float(s.abs().max())
        assert float((g.double().cpu() - w).abs().max()) <= lim


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_value_range(dtype):
    """Rows of zeros, the smallest and largest values, a half difference as large as the
    mean (one of the two points is zero) and none at all."""
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    hq, hk, dh = 2, 1, 48
    dt, ncol = _dt(torch, dtype), 4 * 48
    m = _model(fd, hq, hk, dh, dtype)
    base = _pair(torch, 10, ncol, dt, 3, scale=(1.0, 1.0))
    rows_m = [0.0, 1e-30, 1e-6, 1.0, 1.0, 1e15, 1e30, 3e37, 1.0, 0.0]
    rows_d = [0.0, 1e-33, 1e-9, 0.0, 1.0, 1e12, 1e27, 1e34, 1e-12, 1.0]
    sm, sd = (torch.tensor(r, device="cuda")[:, None] for r in (rows_m, rows_d))
    x = (base[0].float() * sm).to(dt), (base[1].float() * sd).to(dt)
    x[1][4] = x[0][4]
    gains = _gains(torch, dh, dt, 5)
    y = _check_forward(torch, m, x, 10, hq, hk, dh, gains, None, what=f"range {dtype}")
    assert all(bool(torch.isfinite(t[:, :(hq + hk) * dh]).all()) for t in y)
    assert all(bool((t[0] == 0).all()) for t in y)
    dy = _pair(torch, 10, ncol, torch.float32, 6)
    for r in range(10):
        xr, dr = (t[r:r + 1].clone() for t in x), tuple(t[r:r + 1].clone() for t in dy)
        _check_backward(torch, m, tuple(xr), dr, 1, hq, hk, dh, gains, None, what=f"range row {r} {dtype}")


def test_no_direction_and_no_difference_give_zero_difference():
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    hq, hk, dh, T = 3, 1, 40, 9
    m = _model(fd, hq, hk, dh, "f32")
    x = _pair(torch, T, (hq + 2 * hk) * dh, torch.float32, 1, scale=(1.0, 0.0))
    dy = _pair(torch, T, (hq + 2 * hk) * dh, torch.float32, 2, scale=(1.0, 0.0))
    gains = _gains(torch, dh, torch.float32, 3, direction=False)
    y = m.qk_forward(x, T, gains=gains, eps=EPS)
    dx, dg = m.qk_backward(dy, T, x=x, gains=gains, eps=EPS)
    assert bool((y[1] == 0).all()) and bool((dx[1] == 0).all()) and all(bool((g == 0).all()) for g in dg)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_non_finite_values_stay_in_their_head(bad):
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    hq, hk, dh, T = 4, 2, 32, 6
    ncol = (hq + 2 * hk) * dh
    m = _model(fd, hq, hk, dh, "bf16")
    x = _pair(torch, T, ncol, torch.bfloat16, 1)
    dy = _pair(torch, T, ncol, torch.float32, 2)
    gains = _gains(torch, dh, torch.bfloat16, 3)
    y0 = m.qk_forward(x, T, gains=gains, eps=EPS)
    dx0, dg0 = m.qk_backward(dy, T, x=x, gains=gains, eps=EPS)
    for ch in range(2):
        xb = tuple(t.clone() for t in x)
        xb[ch][2, dh + 5] = bad                       # token 2, query head 1
        y = m.qk_forward(xb, T, gains=gains, eps=EPS)
        dx, dg = m.qk_backward(dy, T, x=xb, gains=gains, eps=EPS)
        mask = torch.zeros(T, ncol, dtype=torch.bool, device="cuda")
        mask[2, dh:2 * dh] = True
        for a, b in list(zip(y, y0)) + list(zip(dx, dx0)):
            assert bool(torch.isnan(a[mask]).all()) and torch.equal(a[~mask], b[~mask])
        assert bool(torch.isnan(dg[0]).all()) and torch.equal(dg[1], dg0[1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_in_place_strides_and_untouched_memory(dtype):
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    hq, hk, dh, T, S = 6, 2, 56, 15, 5
    dt, ncol = _dt(torch, dtype), 10 * 56
    m = _model(fd, hq, hk, dh, dtype, True, (10, 10, 8))
    gains = _gains(torch, dh, dt, 3)
    pos = torch.randint(0, 99, (3, T), dtype=torch.int32, device="cuda")
    x = _pair(torch, T, ncol, dt, 1)
    dy = _pair(torch, T, ncol, torch.float32, 2)
    y = m.qk_forward(x, S, gains=gains, eps=EPS, positions=pos)
    dx, dg = m.qk_backward(dy, S, x=x, gains=gains, eps=EPS, positions=pos)
    # in place
    z = tuple(t.clone() for t in x)
    r = m.qk_forward(z, S, gains=gains, eps=EPS, positions=pos, out=z)
    assert r is z and all(torch.equal(a, b) for a, b in zip(z, y))
    # mean and half difference as the two halves of one buffer's rows, input and output
    # side by side, rows before and after left alone
    buf = torch.full((T + 2, 4 * ncol + 16), 3.0, dtype=dt, device="cuda")
    xs, ys = (tuple(buf[1:-1, (2 * i + j) * ncol:(2 * i + j + 1) * ncol] for j in range(2)) for i in range(2))
    for a, b in zip(xs, x):
        a.copy_(b)
    m.qk_forward(xs, S, gains=gains, eps=EPS, positions=pos, out=ys)
    assert all(torch.equal(a, b) for a, b in zip(ys, y)) and all(torch.equal(a, b) for a, b in zip(xs, x))
    ys[0].fill_(3.0), ys[1].fill_(3.0)
    m.qk_backward(dy, S, x=xs, gains=gains, eps=EPS, positions=pos, out=ys)
    assert all(torch.equal(a, b) for a, b in zip(ys, dx))
    assert bool((buf[0] == 3).all()) and bool((buf[-1] == 3).all()) and bool((buf[:, 4 * ncol:] == 3).all())
    # gains and positions at odd element offsets
    go = tuple(torch.cat([g[:1], g])[1:] for g in gains)
    po = torch.cat([pos.reshape(-1)[:1], pos.reshape(-1)])[1:]
    assert all(torch.equal(a, b) for a, b in zip(m.qk_forward(x, S, gains=go, eps=EPS, positions=po), y))
    dx2, dg2 = m.qk_backward(dy, S, x=x, gains=go, eps=EPS, positions=po)
    assert all(torch.equal(a, b) for a, b in zip((*dx2, *dg2), (*dx, *dg)))


def test_accumulate_empty_and_repeated_calls():
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    hq, hk, dh, T = 16, 4, 64, 2000
    ncol = (hq + 2 * hk) * dh
    m = _model(fd, hq, hk, dh, "bf16")
    x = _pair(torch, T, ncol, torch.bfloat16, 1)
    dy = _pair(torch, T, ncol, torch.float32, 2)
    gains = _gains(torch, dh, torch.bfloat16, 3)
    sc = m.qk_scratch(1, T)
    sc.fill_(255)                                     # NaN patterns: every row that is read was written
    dx, dg = m.qk_backward(dy, T, x=x, gains=gains, eps=EPS, scratch=sc)
    for _ in range(3):
        sc.fill_(255)
        dx2, dg2 = m.qk_backward(dy, T, x=x, gains=gains, eps=EPS, scratch=sc)
        assert all(torch.equal(a, b) for a, b in zip((*dx, *dg), (*dx2, *dg2)))
    start = tuple(torch.randn(dh, device="cuda") for _ in range(2))
    acc = tuple(t.clone() for t in start)
    m.qk_backward(dy, T, x=x, gains=gains, eps=EPS, gain_grads=acc, accumulate=True, scratch=sc)
    for a, s, g in zip(acc, start, dg):
        # one rounding of the sum, and dg's own
        lim = R.U32 * ((s.double() + g.double()).abs() + g.double().abs()) * 1.01
        assert bool(((a.double() - (s.double() + g.double())).abs() <= lim).all())
    # no tokens: gradients are zero, or what was there
    none = tuple(torch.empty(0, ncol, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    nod = tuple(torch.empty(0, ncol, device="cuda") for _ in range(2))
    assert m.qk_forward(none, 4, gains=gains, eps=EPS)[0].shape == (0, ncol)
    _, z = m.qk_backward(nod, 4, x=none, gains=gains, eps=EPS)
    assert all(bool((t == 0).all()) for t in z)
    kept = tuple(t.clone() for t in start)
    m.qk_backward(nod, 4, x=none, gains=gains, eps=EPS, gain_grads=kept, accumulate=True)
    assert all(torch.equal(a, b) for a, b in zip(kept, start))


@pytest.mark.parametrize("hq,hk,dh,dtype", [(6, 2, 128, "bf16"), (2, 2, 256, "f32")])
def test_long_batch_sums_and_rows(hq, hk, dh, dtype):
    """More tokens than the grid takes at once (several steps per wavefront, a last
    step and a last workgroup that are not full), heads of several tokens in a wavefront
    and of one: every row and the gain gradients."""
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    B, S, ncol = 3, 4099, (hq + 2 * hk) * dh
    T = B * S
    dt = _dt(torch, dtype)
    m = _model(fd, hq, hk, dh, dtype)
    x = _pair(torch, T, ncol, dt, 1)
    dy = _pair(torch, T, ncol, torch.float32, 2)
    gains = _gains(torch, dh, dt, 3)
    y = m.qk_forward(x, S, gains=gains, eps=EPS)
    dx, dg = m.qk_backward(dy, S, x=x, gains=gains, eps=EPS)
    want = R.forward(x, hq, hk, dh, R.angles(dh, BASE, T, S), gains, EPS)
    bound = R.forward_bound(x, hq, hk, dh, R.angles(dh, BASE, T, S), gains, EPS)
    for g, w, b, c in zip(y, want, bound, "md"):
        R.check(g, w, b, f"long y.{c}")
    want, wg = R.backward(x, dy, hq, hk, dh, R.angles(dh, BASE, T, S), gains, EPS)
    bound, bg = R.backward_bound(x, dy, hq, hk, dh, R.angles(dh, BASE, T, S), gains, EPS)
    for g, w, b, c in zip((*dx, *dg), (*want, *wg), (*bound, *bg), ("dx.m", "dx.d", "dq", "dk")):
        R.check(g, w, b, f"long {c}")


def test_backward_is_the_transpose_of_the_forwards_derivative():
    """<w, J d> = <J^T w, d>: with gains that do not move and a small half difference the
    forward's half difference is J d and the backward's mean J^T w at the mean."""
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    hq, hk, dh, T = 4, 2, 96, 37
    ncol = (hq + 2 * hk) * dh
    m = _model(fd, hq, hk, dh, "f32")
    gains = _gains(torch, dh, torch.float32, 3, direction=False)
    x = _pair(torch, T, ncol, torch.float32, 1, scale=(1.0, 1e-4))
    w = _pair(torch, T, ncol, torch.float32, 2, scale=(1.0, 0.0))
    y = m.qk_forward(x, T, gains=gains, eps=EPS)
    dx, _ = m.qk_backward(w, T, x=(x[0], torch.zeros_like(x[1])), gains=gains, eps=EPS)
    a, b = float((w[0].double() * y[1].double()).sum()), float((dx[0].double() * x[1].double()).sum())
    # fp32 roundings of either side (at most 20 steps of the terms' absolute values) and
    # the third-order term, (1e-4)^2 relative
    size = float((w[0].double() * y[1].double()).abs().sum() + (dx[0].double() * x[1].double()).abs().sum())
    say(f"<w, J d> = {a:.9e}, <J^T w, d> = {b:.9e}, terms {size:.3e}")
    assert abs(a - b) <= (20 * R.U32 + 1e-6) * size
    # and the gains' gradient: the half difference along a direction of the gains
    g2 = gains[:2] + _gains(torch, dh, torch.float32, 4)[2:]
    x0 = (x[0], torch.zeros_like(x[1]))
    y2 = m.qk_forward(x0, T, gains=g2, eps=EPS)
    _, dg = m.qk_backward((torch.zeros_like(w[0]), w[0]), T, x=x0, gains=gains, eps=EPS)
    # dy = (0, w): the half difference of the gain gradient is <w, dy/dg>, over eps
    a = float((w[0].double() * y2[1].double()).sum())
    b = sum(float((d.double() * v.double()).sum()) for d, v in zip(dg, g2[2:])) * EPS * EPS
    size = float((w[0].double() * y2[1].double()).abs().sum())
    assert abs(a - b) <= 40 * R.U32 * size


def test_offsets_past_32_bits():
    """2^20 + 5 tokens of 2048 columns (2^31 elements and more), and three rows 2^30
    elements apart: rows are independent, so their bits are those of a small call."""
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    hq, hk, dh = 8, 4, 128
    ncol, T = 2048, 2 ** 20 + 5
    m = _model(fd, hq, hk, dh, "bf16")
    gains = _gains(torch, dh, torch.bfloat16, 3)
    g = torch.Generator(device="cuda").manual_seed(1)
    block = 2 ** 16 + 1
    part = [torch.randn(block, ncol, device="cuda", generator=g) for _ in range(2)]
    x = tuple(torch.empty(T, ncol, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    dy = tuple(torch.empty(T, ncol, device="cuda") for _ in range(2))
    for i in range(0, T, block):
        n = min(block, T - i)
        for k, s in enumerate((1.0, EPS)):
            x[k][i:i + n] = (part[k][:n] * s).roll(i // block, 1).to(torch.bfloat16)
            dy[k][i:i + n] = (part[1 - k][:n] * s).roll(i // block, 1)
    pos = torch.randint(0, 1000, (1, T), dtype=torch.int32, device="cuda", generator=g)
    y = m.qk_forward(x, T, gains=gains, eps=EPS, positions=pos)
    dx, dg = m.qk_backward(dy, T, x=x, gains=gains, eps=EPS, positions=pos)
    for a, b in ((0, 40), (2 ** 19, 2 ** 19 + 33), (T - 70, T)):
        p = pos[:, a:b].contiguous()
        ys = m.qk_forward(tuple(t[a:b] for t in x), b - a, gains=gains, eps=EPS, positions=p)
        dxs, _ = m.qk_backward(tuple(t[a:b] for t in dy), b - a, x=tuple(t[a:b] for t in x), gains=gains, eps=EPS, positions=p)
        for big, small in zip((*y, *dx), (*ys, *dxs)):
            assert torch.equal(big[a:b], small)
    # the gain gradients as a sum over calls: each part and the whole are off by 11
    # roundings of the terms' absolute values, which the signs' cancellation leaves
    # well below 1e-3 of the random sums' size
    acc = [torch.zeros(dh, dtype=torch.float64, device="cuda") for _ in range(2)]
    for a in range(0, T, 2 ** 18):
        b = min(T, a + 2 ** 18)
        _, d = m.qk_backward(tuple(t[a:b] for t in dy), b - a, x=tuple(t[a:b] for t in x), gains=gains, eps=EPS,
                             positions=pos[:, a:b].contiguous())
        for k in range(2):
            acc[k] += d[k].double()
    for k in range(2):
        assert float((dg[k].double() - acc[k]).norm()) <= 1e-3 * float(acc[k].norm())
    del x, dy, y, dx, part
    # rows far apart
    ld = 2 ** 30
    buf = torch.zeros(2 * ld + 4 * ncol, dtype=torch.bfloat16, device="cuda")
    far = [torch.as_strided(buf, (3, ncol), (ld, 1), j * ncol) for j in range(4)]
    xs = _pair(torch, 3, ncol, torch.bfloat16, 5)
    for a, b in zip(far, xs):
        a.copy_(b)
    m.qk_forward(tuple(far[:2]), 3, gains=gains, eps=EPS, out=tuple(far[2:]))
    want = m.qk_forward(xs, 3, gains=gains, eps=EPS)
    assert all(torch.equal(a, b) for a, b in zip(far[2:], want))


@pytest.mark.parametrize("hq,hk,dh", [(3, 1, 24), (5, 5, 48), (9, 3, 72), (17, 1, 96), (3, 3, 144), (2, 1, 168), (6, 2, 192)])
def test_widths_of_twelves(hq, hk, dh):
    """bf16 heads that divide into six pairs per lane."""
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    for norm in (True, False):
        m = _model(fd, hq, hk, dh, "bf16", norm)
        for i, (B, S, pad) in enumerate([(1, 1, 0), (3, 7, 24), (1, 257, 8), (70, 1, 0)]):
            x = _pair(torch, B * S, (hq + 2 * hk) * dh, torch.bfloat16, 40 + i, pad)
            gains = _gains(torch, dh, torch.bfloat16, 50 + i, direction=i != 1) if norm else None
            what = f"{hq}/{hk} heads of {dh}, {B}x{S}{' norm' if norm else ''}"
            say(what)
            _check_forward(torch, m, x, S, hq, hk, dh, gains, None, what=what)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("norm", [True, False])
@pytest.mark.parametrize("hq,hk,dh", [(64, 64, 16), (5, 1, 64), (40, 8, 72), (32, 8, 80), (16, 4, 128), (14, 2, 136), (12, 4, 144),
                                      (12, 4, 192), (4, 1, 256)])
def test_runs_of_tokens(hq, hk, dh, norm, dtype):
    """Batches long enough for several tokens (or groups of them) per wavefront, the last
    run cut short: rows are independent, so their bits are those of a shorter call."""
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    T, ncol, n = 64 * 173 + 5, (hq + 2 * hk) * dh, 64 * 7   # (parts of whole groups of tokens)
    dt = _dt(torch, dtype)
    m = _model(fd, hq, hk, dh, dtype, norm)
    g = torch.Generator(device="cuda").manual_seed(dh)
    gains = _gains(torch, dh, dt, 3) if norm else None
    x = tuple((torch.randn(T, ncol, device="cuda", generator=g) * s).to(dt) for s in (1.0, EPS))
    dy = tuple(torch.randn(T, ncol, device="cuda", generator=g) * s for s in (1.0, EPS))
    pos = torch.randint(0, 5000, (1, T), dtype=torch.int32, device="cuda", generator=g)
    say(f"{hq}/{hk} heads of {dh}, {T} tokens {dtype}{' norm' if norm else ''}")
    y = m.qk_forward(x, T, gains=gains, eps=EPS, positions=pos)
    dx = m.qk_backward(dy, T, x=x if norm else None, gains=gains, eps=EPS, positions=pos)
    dx = dx[0] if norm else dx
    for a in (*range(0, T - n, n), T - n):
        b = a + n
        p = pos[:, a:b].contiguous()
        ys = m.qk_forward(tuple(t[a:b] for t in x), b - a, gains=gains, eps=EPS, positions=p)
        ds = m.qk_backward(tuple(t[a:b] for t in dy), b - a, x=tuple(t[a:b] for t in x) if norm else None, gains=gains, eps=EPS,
                           positions=p)
        for big, small in zip((*y, *dx), (*ys, *(ds[0] if norm else ds))):
            assert torch.equal(big[a:b], small), (a, b)


def test_more_wavefronts_than_a_launch_holds():
    """2^21 + 2^12 tokens of 62 + 2 heads of 136, in place: at one token per
    wavefront 32 of them a token, 2^26 and more, above the 2^32 threads of a launch."""
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    hq, hk, dh = 62, 2, 136
    S, B = 2 ** 12, 2 ** 9 + 1
    T, ncol = S * B, (hq + 2 * hk) * dh
    gc.collect()   # what earlier tests left
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 4 * T * ncol + 2 ** 32:
        pytest.skip("80 GB of free memory needed")
    m = _model(fd, hq, hk, dh, "bf16", norm=False)
    x = tuple(torch.zeros(T, ncol, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    rows = _pair(torch, 2 * S, ncol, torch.bfloat16, 9)
    want = m.qk_forward(rows, S)
    at = (0, T // 2 // S * S, T - 2 * S)
    for a in at:
        for t, r in zip(x, rows):
            t[a:a + 2 * S] = r
    y = m.qk_forward(x, S, out=x)
    for a in at:
        assert all(torch.equal(t[a:a + 2 * S], w) for t, w in zip(y, want)), a
    del x, y
    torch.cuda.empty_cache()


def test_shared_inputs_and_plain_positions():
    """One tensor as mean and half difference (one point is zero), one gain for queries
    and keys, given positions on a model with one axis."""
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    hq, hk, dh, T = 4, 2, 64, 21
    ncol = (hq + 2 * hk) * dh
    m = _model(fd, hq, hk, dh, "f32")
    t = _pair(torch, T, ncol, torch.float32, 1)[0]
    g = _gains(torch, dh, torch.float32, 2)
    gains = (g[0], g[0], g[2], g[2])
    pos = torch.randint(-30, 30, (1, 3, 7), dtype=torch.int32, device="cuda")
    _check_forward(torch, m, (t, t), 7, hq, hk, dh, gains, pos, what="one tensor")
    dy = _pair(torch, T, ncol, torch.float32, 3)
    _check_backward(torch, m, (t, t), (dy[0], dy[0]), 7, hq, hk, dh, gains, pos, what="one tensor")


def test_calls_on_two_streams_at_once():
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    hq, hk, dh, T = 8, 8, 64, 4000
    ncol = (hq + 2 * hk) * dh
    work = []
    for i in range(2):
        s = torch.cuda.Stream()
        m = _model(fd, hq, hk, dh, "bf16", stream=s.cuda_stream)
        x = _pair(torch, T, ncol, torch.bfloat16, 10 * i)
        dy = _pair(torch, T, ncol, torch.float32, 10 * i + 1)
        gains = _gains(torch, dh, torch.bfloat16, 10 * i + 2)
        with torch.cuda.stream(s):
            want = m.qk_backward(dy, T, x=x, gains=gains, eps=EPS)
        torch.cuda.synchronize()
        work.append((s, m, x, dy, gains, want))
    got = [[], []]
    for _ in range(10):
        for i, (s, m, x, dy, gains, _) in enumerate(work):
            with torch.cuda.stream(s):
                got[i].append(m.qk_backward(dy, T, x=x, gains=gains, eps=EPS))
    torch.cuda.synchronize()
    for i in range(2):
        wdx, wdg = work[i][5]
        for dx, dg in got[i]:
            assert all(torch.equal(a, b) for a, b in zip((*dx, *dg), (*wdx, *wdg)))


def test_rotation_and_back():
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    hq, hk, dh, T = 3, 1, 128, 50
    m = _model(fd, hq, hk, dh, "f32", False, (22, 21, 21), True)
    x = _pair(torch, T, (hq + 2 * hk) * dh, torch.float32, 1)
    pos = torch.randint(-1000, 1000, (3, T), dtype=torch.int32, device="cuda")
    back = m.qk_backward(m.qk_forward(x, T, positions=pos), T, positions=pos)
    for a, b in zip(back, x):
        # two rotations of 3 roundings each, terms up to |x_i| + |x_j| twice
        assert float((a - b).abs().max()) <= 6 * R.U32 * 4 * float(b.abs().max())


def test_graph_replays_and_other_streams():
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    hq, hk, dh, S = 8, 2, 128, 300
    ncol = (hq + 2 * hk) * dh
    side = torch.cuda.Stream()
    m = _model(fd, hq, hk, dh, "bf16", True, (24, 20, 20), stream=side.cuda_stream)
    eager = _model(fd, hq, hk, dh, "bf16", True, (24, 20, 20))
    gains = _gains(torch, dh, torch.bfloat16, 3)
    x = _pair(torch, S, ncol, torch.bfloat16, 1)
    dy = _pair(torch, S, ncol, torch.float32, 2)
    pos = torch.randint(0, 5000, (3, S), dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError, match="stream"):
        m.qk_forward(x, S, gains=gains, eps=EPS, positions=pos)
    side.wait_stream(torch.cuda.current_stream())
    graphs, outs = [], []
    with torch.cuda.stream(side):
        with pytest.raises(ValueError, match="stream"):
            eager.qk_forward(x, S, gains=gains, eps=EPS, positions=pos)
        # two graphs, each with buffers of its own
        for _ in range(2):
            y = tuple(torch.empty_like(t) for t in x)
            dx = tuple(torch.empty_like(t) for t in x)
            dg = tuple(torch.empty(dh, device="cuda") for _ in range(2))
            sc = m.qk_scratch(1, S)
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=side):
                m.qk_forward(x, S, gains=gains, eps=EPS, positions=pos, out=y)
                m.qk_backward(dy, S, x=x, gains=gains, eps=EPS, positions=pos, out=dx, gain_grads=dg, scratch=sc)
            graphs.append(g)
            outs.append((*y, *dx, *dg, sc))
    torch.cuda.synchronize()
    for step in range(4):
        with torch.no_grad():
            for t, s in zip(x + dy, range(4)):
                t.copy_(torch.randn(t.shape, generator=torch.Generator().manual_seed(100 * step + s)) * (1.0 if s % 2 == 0 else EPS))
            pos.add_(17)
        torch.cuda.synchronize()
        want = (*eager.qk_forward(x, S, gains=gains, eps=EPS, positions=pos),)
        wdx, wdg = eager.qk_backward(dy, S, x=x, gains=gains, eps=EPS, positions=pos)
        torch.cuda.synchronize()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for o in outs:
            assert all(torch.equal(a, b) for a, b in zip(o[:6], (*want, *wdx, *wdg))), step


def test_binding_refusals_on_the_device():
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    m = _model(fd, 2, 1, 32, "bf16", True, (6, 5, 5))
    x = _pair(torch, 4, 128, torch.bfloat16, 1)
    gains = _gains(torch, 32, torch.bfloat16, 2)
    with pytest.raises(fd.FdhError, match="gains are required"):
        m.qk_forward(x, 4)
    with pytest.raises(ValueError, match="divide"):
        m.qk_forward(x, 3, gains=gains)
    with pytest.raises(ValueError, match="divide"):
        m.qk_forward(x, 0, gains=gains)
    with pytest.raises(ValueError, match="positions"):
        m.qk_forward(x, 4, gains=gains, positions=torch.zeros(2, 4, dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError, match="positions"):
        m.qk_forward(x, 4, gains=gains, positions=torch.zeros(3, 4, dtype=torch.int64, device="cuda"))
    with pytest.raises(ValueError, match="device"):
        m.qk_forward(x, 4, gains=gains, positions=torch.zeros(3, 4, dtype=torch.int32))
    with pytest.raises(ValueError, match="dtype"):
        m.qk_forward(tuple(t.float() for t in x), 4, gains=gains)
    with pytest.raises(ValueError, match="device"):
        m.qk_forward((x[0], x[1].cpu()), 4, gains=gains)
    with pytest.raises(ValueError, match="device"):
        m.qk_forward(x, 4, gains=(*gains[:3], gains[3].cpu()))
    with pytest.raises(ValueError, match="gains"):
        m.qk_forward(x, 4, gains=(gains[0].float(), *gains[1:]))
    with pytest.raises(fd.FdhError, match="overlaps"):
        m.qk_forward(x, 4, gains=gains, out=(x[1], x[0]))
    with pytest.raises(fd.FdhError, match="eps"):
        m.qk_forward(x, 4, gains=gains, eps=0.0)
    dy = _pair(torch, 4, 128, torch.float32, 3)
    with pytest.raises(ValueError, match="needs x"):
        m.qk_backward(dy, 4, gains=gains)
    with pytest.raises(ValueError, match="gain_grads"):
        m.qk_backward(dy, 4, x=x, gains=gains, accumulate=True)
    with pytest.raises(ValueError, match="scratch"):
        m.qk_backward(dy, 4, x=x, gains=gains, scratch=torch.empty(1 << 16, dtype=torch.uint8, device="cuda")[::2])
    with pytest.raises(fd.FdhError, match="scratch"):
        m.qk_backward(dy, 4, x=x, gains=gains, scratch=torch.empty(8, dtype=torch.uint8, device="cuda"))
