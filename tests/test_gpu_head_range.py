"""Beyond the range of the logits' half differences that the vocabulary loss is documented for: a row's results are
either within the bounds that hold inside it, or NaN, never another number; the HVP names the cause."""
import pytest

from tests import ends_points_ref as P
from tests import ends_ref as R
from tests.gpu_util import need_gpu, say

pytestmark = pytest.mark.gpu


def _shifted(torch, T, V, d, dtype, shift, seed):
    """Logits of a few units whose half differences are all within 2 of shift: beyond the range by a shift that the
    softmax does not see."""
    g = torch.Generator().manual_seed(seed)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    xm, xd = torch.randn(T, d, generator=g), 0.1 * torch.randn(T, d, generator=g)
    wm, wd = torch.randn(V, d, generator=g) * (1.0 / d ** 0.5), torch.zeros(V, d)
    xm[:, 0], xd[:, 0], wm[:, 0] = 0.0, shift, 1.0
    tgt = torch.randint(0, V, (T,), generator=g)
    return (xm.to(dt), xd.to(dt)), (wm.to(dt), wd.to(dt)), tgt.to(torch.int32)


@pytest.mark.parametrize("dtype,reach", [("bf16", 20.0), ("bf16", 34.0), ("bf16", 40.0), ("bf16", 43.0), ("bf16", 44.0), ("bf16", 47.0), ("bf16", 90.0),
                                         ("f32", 200.0), ("f32", 340.0), ("f32", 353.0), ("f32", 360.0), ("f32", 600.0)])
@pytest.mark.parametrize("T", [1, 20, 70, 300])
def test_a_row_is_right_or_not_a_number(T, dtype, reach):
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    V, d = 2056, 64
    m = fd.Model("llama", 0, d, 1, 1, 8, V, 2, dtype)
    for kind in ("shifted", "spread"):
        x, w, tgt = _shifted(torch, T, V, d, dtype, reach, T) if kind == "shifted" else P.inputs(T, V, d, dtype, reach, T, ignore=0.0)
        what = f"{kind} T {T} {dtype} half differences {reach}"
        args = (x, w, tgt, 1.0, 1.0)
        want, lim = R.head(*args), P.bound(*args)
        for piece in (0, 512):
            dx = tuple(torch.empty(T, d, device="cuda") for _ in range(2))
            loss, dx, dw = m.head_grad(tuple(a.cuda() for a in x), tuple(a.cuda() for a in w), tgt.cuda(), eps=1.0, piece=piece, dx=dx,
                                       dw=torch.empty(V, d, device="cuda"))
            torch.cuda.synchronize()
            nan = [torch.isnan(a.cpu()).reshape(T, -1).any(1) for a in (*loss, *dx)]
            say(f"{what} piece {piece}: {int(nan[0].sum())} rows NaN")
            assert all(torch.equal(a, nan[0]) for a in nan)
            if reach <= (30 if dtype == "bf16" else 300):
                assert not bool(nan[0].any())
            ok = ~nan[0]
            for a, v, b, c in zip((*loss, *dx), (*want[0], *want[1]), (*lim[0], *lim[1]), ("loss.m", "loss.d", "dx.m", "dx.d")):
                R.check(a.cpu()[ok], v[ok], b[ok], f"{what} {c}")
            if bool(nan[0].any()):
                assert bool(torch.isnan(dw).any())
            else:
                R.check(dw, want[2], lim[2], f"{what} dw")


def test_hvp_says_why():
    """A step far too long, in pieces: refused, and the message names the range; whole logits take it.  The direction
    adds the same row to every word's, so that a token's logits move together, by 6 sqrt(128) = 68 in the mean
    square."""
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    V, d = 1000, 128
    said = []
    for piece in (0, 256):
        m = fd.Model("llama", 0, d, 1, 1, 8, V, 64, "bf16")
        m.set_vocab_piece(piece)
        m.set_workspace(1, 64)
        th, v = m.init_params(1), torch.zeros(m.num_params, device="cuda")
        head = next(e for e in m.layout() if e.name == "head")
        v[head.offset:head.offset + head.numel] = 1.0
        try:
            assert bool(torch.isfinite(m.hvp(th, v, 6.0, m.make_tokens(1, 64, 2))).all())
            said.append("")
        except fd.FdhError as e:
            said.append(str(e))
    assert said[0] == "" and "half differences" in said[1], said
