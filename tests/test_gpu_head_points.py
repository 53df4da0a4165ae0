"""The loss over the vocabulary where the two points are apart in x and in w alike: the documented
loss and gradients, for every number of rows, over the documented range of the logits' half
differences, with nothing left out."""
import pytest

from tests import ends_points_ref as P
from tests import ends_ref as R
from tests.gpu_util import need_gpu, say

pytestmark = pytest.mark.gpu

REACH = [("bf16", 0.5), ("bf16", 1.5), ("bf16", 5.0), ("bf16", 28.0), ("f32", 0.1), ("f32", 0.5), ("f32", 1.5), ("f32", 5.0), ("f32", 28.0),
         ("f32", 290.0)]


def _model(fd, V, d, dtype, **kw):
    return fd.Model("llama", 0, d, 1, 1, 8, V, 2, dtype, **kw)


def _run(torch, fd, T, V, d, dtype, reach, piece, seed, eps=1e-2):
    what = f"T {T} V {V} d {d} {dtype} half differences {reach} piece {piece}"
    say(what)
    m = _model(fd, V, d, dtype)
    x, w, tgt = P.inputs(T, V, d, dtype, reach, seed)
    gx, gw, gt = tuple(a.cuda() for a in x), tuple(a.cuda() for a in w), tgt.cuda()
    dx = tuple(torch.full((T, d), 3.0, device="cuda") for _ in range(2))
    got = m.head_grad(gx, gw, gt, scale=1.0 / T, eps=eps, piece=piece, dx=dx, dw=torch.full((V, d), 3.0, device="cuda"))
    alone = m.head_loss(gx, gw, gt, piece=piece)
    torch.cuda.synchronize()
    P.check(got, x, w, tgt, 1.0 / T, eps, what)
    P.check((alone, None, None), x, w, tgt, 1.0 / T, eps, what + " loss alone")


@pytest.mark.parametrize("dtype,reach", REACH)
@pytest.mark.parametrize("T", [1, 8, 9, 32, 33, 130, 300])
def test_every_number_of_rows(T, dtype, reach):
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    for piece in (0, 256):
        _run(torch, fd, T, 520, 64, dtype, reach, piece, T)


@pytest.mark.parametrize("dtype,reach", [("bf16", 5.0), ("f32", 0.5), ("f32", 5.0)])
@pytest.mark.parametrize("T,V,d,piece", [(65, 12296, 72, 0), (130, 12296, 264, 0), (300, 12296, 136, 0), (300, 12296, 136, 6144), (520, 24584, 24, 0),
                                         (2047, 1032, 72, 0), (40, 1000, 1032, 512)])
def test_every_tile(T, V, d, piece, dtype, reach):
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    _run(torch, fd, T, V, d, dtype, reach, piece, T)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_row_among_others(dtype):
    """What a row gives does not hang on how many stand beside it: the first 8 rows of ever larger
    batches, each within the bounds of the same statement."""
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    V, d = 1032, 64
    x, w, tgt = P.inputs(400, V, d, dtype, 5.0, 7, ignore=0.0)
    gw = tuple(a.cuda() for a in w)
    m = _model(fd, V, d, dtype)
    head = (tuple(a[:8] for a in x), w, tgt[:8])
    want, lim = R.head(*head, 1.0, 1e-2), P.bound(*head, 1.0, 1e-2)
    for T in (8, 9, 16, 32, 33, 64, 65, 128, 129, 400):
        dx = tuple(torch.empty(T, d, device="cuda") for _ in range(2))
        loss, dx, _ = m.head_grad(tuple(a[:T].cuda() for a in x), gw, tgt[:T].cuda(), eps=1e-2, dx=dx, dw=torch.empty(V, d, device="cuda"))
        torch.cuda.synchronize()
        for a, v, b, c in zip((*loss, *dx), (*want[0], *want[1]), (*lim[0], *lim[1]), ("loss.m", "loss.d", "dx.m", "dx.d")):
            R.check(a[:8], v, b, f"T {T} {dtype} {c}")
