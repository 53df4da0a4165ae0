"""The vocabulary loss at the ends of its documented sizes: 2^20 rows, widths to 2^16, the smallest vocabulary and the
largest, and large products repeated bit for bit."""
import pytest

from tests import ends_points_ref as P
from tests import ends_ref as R
from tests.gpu_util import need_gpu, say

pytestmark = pytest.mark.gpu

EPS = 1e-2


def _model(fd, V, d, dtype):
    return fd.Model("llama", 0, d, 1, 1, 8, V, 2, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,V,d,piece", [(1, 8, 65536, 0), (1, 1032, 65536, 0), (8, 520, 65528, 0), (9, 520, 65536, 256), (40, 520, 65528, 0), (33, 8, 8, 0),
                                         (5, 262136, 8, 0), (40, 262136, 16, 0), (40, 262136, 16, 100000)])
def test_widths_and_vocabularies(T, V, d, piece, dtype):
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    say(f"{dtype} T {T} V {V} d {d} piece {piece}")
    m = _model(fd, V, d, dtype)
    x, w, tgt = P.inputs(T, V, d, dtype, 0.5, T + V)
    if bool((tgt == R.IGNORE).all()):
        tgt[0] = V - 1
    dx = tuple(torch.empty(T, d, device="cuda") for _ in range(2))
    got = m.head_grad(tuple(a.cuda() for a in x), tuple(a.cuda() for a in w), tgt.cuda(), scale=1.0 / T, eps=EPS, piece=piece, dx=dx,
                      dw=torch.empty(V, d, device="cuda"))
    torch.cuda.synchronize()
    P.check(got, x, w, tgt, 1.0 / T, EPS, "")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V,d,piece", [(72, 24, 0), (2056, 8, 0), (2056, 8, 1024)])
def test_most_rows(V, d, piece, dtype):
    """2^20 of them: some rows against the statement, dw against the definition in float64 on the device."""
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    T = 1 << 20
    say(f"{dtype} T {T} V {V} d {d} piece {piece}")
    m = _model(fd, V, d, dtype)
    x, w, tgt = P.inputs(4096, V, d, dtype, 0.5, 3, ignore=0.2)
    many = torch.randint(0, 4096, (T,), generator=torch.Generator().manual_seed(4))
    gx, gw, gt = tuple(a[many].cuda() for a in x), tuple(a.cuda() for a in w), tgt[many].cuda()
    dx = tuple(torch.empty(T, d, device="cuda") for _ in range(2))
    loss, dx, dw = m.head_grad(gx, gw, gt, scale=1.0, eps=EPS, piece=piece, dx=dx, dw=torch.empty(V, d, device="cuda"))
    torch.cuda.synchronize()
    want, lim = R.head(x, w, tgt, 1.0, EPS), P.bound(x, w, tgt, 1.0, EPS)
    rows = torch.cat([torch.arange(300), torch.arange(T // 2 - 150, T // 2 + 150), torch.arange(T - 300, T)])
    for a, v, b, c in zip((*loss, *dx), (*want[0], *want[1]), (*lim[0], *lim[1]), ("loss.m", "loss.d", "dx.m", "dx.d")):
        R.check(a[rows.cuda()], v[many[rows]], b[many[rows]], c)
    n = torch.bincount(many, minlength=4096).to(torch.float64)[:, None]
    live = (tgt != R.IGNORE)[:, None].double()
    at = []
    for s in (1, -1):
        a, b = R.f64(x[0]) + s * R.f64(x[1]), R.f64(w[0]) + s * R.f64(w[1])
        p = torch.softmax(a @ b.T, -1)
        p[torch.arange(4096), tgt.long().clamp(min=0)] -= 1.0
        at.append((p * live * n).T @ a)
    want = (at[0] - at[1]) / (2 * EPS)
    # beside the limit of a batch: repeated rows repeat their roundings, and a sum of 2^20 terms in fp32 has 2^10 of
    # them in a row (its parts' and its steps' alike), each half a step of a partial sum
    assert float(torch.linalg.norm(R.f64(dw) - want) / torch.linalg.norm(want)) <= P.whole_limit(x, w) + 2.0 ** 10 * P.U


@pytest.mark.parametrize("dtype,T,V,d,piece", [("bf16", 8192, 32000, 2048, 0), ("bf16", 2047, 32000, 1024, 8192), ("f32", 2047, 8192, 512, 0), ("f32", 4096, 8192, 64, 0)])
def test_the_same_bits_again(dtype, T, V, d, piece):
    """Calls after one another, other work between them and scratch full of other values."""
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    m = _model(fd, V, d, dtype)
    g = torch.Generator(device="cuda").manual_seed(5)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    x = tuple((s * torch.randn(T, d, device="cuda", generator=g)).to(dt) for s in (1.0, 1e-3))
    w = tuple((s * 2 / d ** 0.5 * torch.randn(V, d, device="cuda", generator=g)).to(dt) for s in (1.0, 1e-3))
    tgt = torch.randint(0, V, (T,), device="cuda", dtype=torch.int32, generator=g)
    tgt[::7] = R.IGNORE
    scratch = m.head_scratch(T, piece)
    first = None
    for k in range(4):
        scratch.fill_((0, 255, 127, 60)[k])
        got = m.head_grad(x, w, tgt, scale=1.0 / T, eps=1e-3, piece=piece, scratch=scratch)
        got = (*got[0], *got[1], got[2])
        torch.cuda.synchronize()
        if first is None:
            first = got
        assert all(torch.equal(a, b) for a, b in zip(first, got))
        del got
        (x[0].float() @ w[0][:512].float().T).sum().item()
