"""Every way that the vocabulary loss may take, each asserted to be the one taken: both element types, every
tile in both passes, and rows put in order in fp32 models."""
import pytest

from tests import ends_points_ref as P
from tests import ends_ref as R
from tests import head_routes as H
from tests.gpu_util import need_gpu, say

pytestmark = pytest.mark.gpu

EPS = 1e-2


def _model(fd, V, d, dtype):
    return fd.Model("llama", 0, d, 1, 1, 8, V, 2, dtype)


@pytest.mark.parametrize("dtype,T,V,d,piece,want", H.WAYS)
def test_every_way(dtype, T, V, d, piece, want):
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    m = _model(fd, V, d, dtype)
    H.expect(fd, m, T, piece, want)
    for reach, ignore in ((0.5, 0.3), (3.0, 0.0)):
        what = f"{dtype} T {T} V {V} d {d} piece {piece} half differences {reach}"
        say(what)
        x, w, tgt = P.inputs(T, V, d, dtype, reach, T + piece, ignore)
        pad = tuple(torch.full((T, d + 8), 5.0, dtype=a.dtype, device="cuda") for a in x)
        for a, b in zip(pad, x):
            a[:, :d] = b.cuda()
        # what stands in rows without a target and behind a row's end takes no part
        for a in pad:
            a[:, :d][(tgt == R.IGNORE).cuda()] = float("nan")
        gx, gw, gt = tuple(a[:, :d] for a in pad), tuple(a.cuda() for a in w), tgt.cuda()
        base = torch.randn(V, d, generator=torch.Generator().manual_seed(3))
        dx = tuple(torch.full((T, d), 3.0, device="cuda") for _ in range(2))
        got = m.head_grad(gx, gw, gt, scale=0.25, eps=EPS, piece=piece, dx=dx, dw=torch.full((V, d), 3.0, device="cuda"))
        more = m.head_grad(gx, gw, gt, scale=0.25, eps=EPS, piece=piece, dx=tuple(torch.empty_like(a) for a in dx), dw=base.cuda(), accumulate=True)
        alone = m.head_loss(gx, gw, gt, piece=piece)
        torch.cuda.synchronize()
        args = (x, w, tgt, 0.25, EPS)
        P.check(got, *args, what)
        P.check((alone, None, None), *args, what + " loss alone")
        ww, bw = R.head(*args)[2], P.bound(*args)[2]
        R.check(more[2], ww + R.f64(base), bw + 2.0 ** -23 * (R.f64(base).abs() + ww.abs()), what + " added")
        assert all(torch.equal(a, b) for a, b in zip((*more[0], *more[1]), (*got[0], *got[1])))


@pytest.mark.parametrize("T,V,d,piece,want", H.ORDERED)
def test_rows_in_order_in_fp32(T, V, d, piece, want):
    """Rows without a target hold NaN and are not multiplied: the others give the bits that they give where every
    row has a target, and dw is the definition's over them."""
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    m = _model(fd, V, d, "f32")
    H.expect(fd, m, T, piece, want)
    x, w, full = (tuple(a.cuda() for a in t) if isinstance(t, tuple) else t.cuda() for t in P.inputs(T, V, d, "f32", 0.5, 21, ignore=0.0))
    wide = tuple(torch.full((T, d + 4), 5.0, device="cuda") for _ in x)

    def run(tgt, none):
        for a, b in zip(wide, x):
            a[:, :d] = torch.where(none[:, None], torch.full_like(b, float("nan")), b)
        dx = tuple(torch.full((T, d), 5.0, device="cuda") for _ in range(2))
        got = m.head_grad(tuple(a[:, :d] for a in wide), w, tgt, scale=1.0 / T, eps=EPS, piece=piece, dx=dx, dw=torch.full((V, d), 5.0, device="cuda"))
        torch.cuda.synchronize()
        return got

    def definition(tgt, live):
        at = []
        for sign in (1.0, -1.0):
            a, b = x[0].double() + sign * x[1].double(), w[0].double() + sign * w[1].double()
            dw, loss, dx = torch.zeros_like(b), [], []
            for i in range(0, T, 1024):
                r = slice(i, i + 1024)
                k = live[r].nonzero()[:, 0]
                lp = torch.log_softmax(a[r] @ b.T, -1)
                y = tgt[r][k].long()
                l = torch.zeros(lp.shape[0], device="cuda", dtype=torch.float64)
                l[k] = -lp[k, y]
                p = lp.exp_()
                p[k, y] -= 1.0
                p *= live[r][:, None].double() / T
                loss.append(l)
                dx.append(p @ b)
                dw += p.T @ a[r]
            at.append((torch.cat(loss), torch.cat(dx), dw))
        (lp, xp, wp), (lm, xm, wm) = at
        return ((lp + lm) / 2, (lp - lm) / 2), ((xp + xm) / 2, (xp - xm) / 2), (wp - wm) / (2 * EPS)

    whole = run(full, torch.zeros(T, dtype=torch.bool, device="cuda"))
    lim = P.whole_limit(tuple(a[:512] for a in x), w)
    t = torch.arange(T)
    g = torch.Generator().manual_seed(22)
    masks = {"none": t < 0, "scattered": torch.rand(T, generator=g) < 0.3, "most": torch.rand(T, generator=g) < 0.95, "the end": t >= T // 3,
             "the start": t < T - 7, "all but one": t != T // 2, "all": t >= 0}
    for name, none in masks.items():
        say(f"T {T} V {V} d {d} piece {piece} without a target: {name}")
        none = none.cuda()
        tgt = torch.where(none, torch.full_like(full, R.IGNORE), full)
        loss, dx, dw = run(tgt, none)
        for a, b in zip((*loss, *dx), (*whole[0], *whole[1])):
            assert torch.equal(a[~none], b[~none]) and float(a[none].abs().sum()) == 0.0
        if name == "all":
            assert float(dw.abs().max()) == 0.0
            continue
        want = definition(tgt, ~none)
        for a, v in zip((*loss, *dx, dw), (*want[0], *want[1], want[2])):
            assert float(torch.linalg.norm(a.double() - v) / torch.linalg.norm(v)) <= lim


@pytest.mark.parametrize("B,S,piece,tile", [(1, 64, 2048, (64, 64)), (1, 64, 32000, (64, 128)), (2, 128, 8192, (64, 128)), (2, 128, 16384, (128, 128)),
                                            (2, 128, 32000, (256, 128)), (8, 64, 16384, (256, 128)), (1, 24, 4096, (32, 128)), (1, 8, 4096, (32, 128))])
def test_hvp_in_pieces_of_every_tile(B, S, piece, tile):
    """The tiles without the product of two half differences, which the HVP alone takes: products and losses
    beside those of whole logits (both round the logits' gradient to bf16: half a step each)."""
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    V = 32000
    hv, losses = [], []
    for p in (0, piece):
        m = fd.Model("llama", 1, 128, 2, 2, 256, V, 512, "bf16")
        m.set_vocab_piece(p)
        m.set_workspace(B, S)
        if p:
            r = H.route(fd, m, B * S, p)
            assert (r["rows"], r["columns"]) == tile and r["fused"] and r["keep"] == int(p == V or B * S <= 8)
        th = m.init_params(1)
        hv.append(m.hvp(th, m.random_vector(3), 1e-3, m.make_tokens(B, S, 2, "uniform")))
        losses.append(m.last_losses())
    err = float((hv[0] - hv[1]).double().norm() / hv[0].double().norm())
    say(f"T {B * S} piece {piece}: {err:.2e}")
    assert err < 2 * 2.0 ** -8
    assert all(abs(a - b) < 1e-6 * abs(a) for a, b in zip(*losses))
