"""The loss over the vocabulary in pieces (fdh_head_loss, fdh_head_grad) against the float64
statement of tests/ends_ref.py: one row to some hundred, odd sizes, vocabularies below and
beyond a piece, strides, rows without a target (with NaN in them), all of them, targets
outside the vocabulary, points far apart, accumulation, repeated calls, graphs, streams."""
import pytest

from tests import ends_ref as R
from tests.gpu_util import need_gpu, say

pytestmark = pytest.mark.gpu

EPS = 1e-3


def _dt(torch, dtype):
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def _model(fd, V, d, dtype, **kw):
    return fd.Model("llama", 0, d, 1, 1, 8, V, 2, dtype, **kw)


def _case(torch, T, V, d, dtype, seed, pad=0, ignore=0.2, half=EPS, size=2.0):
    g = torch.Generator().manual_seed(seed)
    dt = _dt(torch, dtype)

    def rows(n, s, p):
        full = torch.full((n, d + p), 7.0, dtype=dt)
        full[:, :d] = (torch.randn(n, d, generator=g) * s).to(dt)
        return full.cuda()[:, :d]

    x = rows(T, 1.0, pad), rows(T, half, pad)
    w = rows(V, size / d ** 0.5, 0), rows(V, half * size / d ** 0.5, 0)
    tgt = torch.randint(0, V, (T,), generator=g)
    tgt[torch.rand(T, generator=g) < ignore] = R.IGNORE
    return x, w, tgt.to(torch.int32).cuda()


SHAPES = [  # T, V, d, pad, piece
    (1, 8, 8, 0, 0), (1, 1000, 72, 0, 0), (1, 2056, 264, 8, 256), (2, 24, 16, 8, 0), (3, 264, 40, 0, 256), (4, 5000, 1040, 0, 0),
    (5, 4104, 2056, 8, 0), (7, 520, 64, 8, 0), (8, 256, 136, 0, 0), (9, 256, 136, 0, 0), (16, 2056, 520, 0, 0), (17, 1032, 328, 16, 512), (31, 1000, 40, 16, 512), (32, 4104, 64, 0, 0),
    (33, 2056, 72, 0, 300), (64, 1024, 256, 0, 256), (65, 640, 512, 0, 0), (130, 2056, 264, 8, 1024), (257, 5000, 128, 0, 0),
    (256, 776, 96, 0, 256), (300, 520, 1032, 0, 0), (600, 1304, 40, 8, 512)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,V,d,pad,piece", SHAPES)
def test_loss_and_gradients(T, V, d, pad, piece, dtype):
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    what = f"T {T} V {V} d {d} piece {piece} {dtype}"
    say(what)
    m = _model(fd, V, d, dtype)
    dt = _dt(torch, dtype)
    for i, ignore in enumerate((0.0, 0.3)):
        x, w, tgt = _case(torch, T, V, d, dtype, T + V + i, pad, ignore)
        scale = 1.0 / T
        dxw = [torch.full((T, d + pad), 3.0, dtype=dt, device="cuda") for _ in range(2)]
        got = m.head_grad(x, w, tgt, scale=scale, eps=EPS, piece=piece, dx=tuple(t[:, :d] for t in dxw))
        loss = m.head_loss(x, w, tgt, piece=piece)
        torch.cuda.synchronize()
        R.check_head(got, x, w, tgt, scale, EPS, what)
        R.check_head((loss, None, None), x, w, tgt, scale, EPS, what + " loss alone")
        assert all(bool((t[:, d:] == 3.0).all()) for t in dxw)
        # the same bits in another call, and float32 gradients
        again = m.head_grad(x, w, tgt, scale=scale, eps=EPS, piece=piece)
        assert torch.equal(again[2], got[2]) and all(torch.equal(a, b) for a, b in zip((*again[0], *again[1]), (*got[0], *got[1])))
        if dtype == "bf16":
            dw = torch.empty(V, d, device="cuda")
            wide = m.head_grad(x, w, tgt, scale=scale, eps=EPS, piece=piece, dw=dw)
            torch.cuda.synchronize()
            R.check_head(wide, x, w, tgt, scale, EPS, what + " in float32")


@pytest.mark.parametrize("T", [77, 5])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_accumulate(dtype, T):
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    V, d = 1032, 72
    m = _model(fd, V, d, dtype)
    x, w, tgt = _case(torch, T, V, d, dtype, 5)
    for piece in (0, 256):
        base = torch.randn(V, d, generator=torch.Generator().manual_seed(1)).cuda()
        dw = base.clone()
        dx = tuple(torch.full((T, d), 9.0, device="cuda") for _ in range(2))
        got = m.head_grad(x, w, tgt, eps=EPS, piece=piece, dx=dx, dw=dw, accumulate=True)
        torch.cuda.synchronize()
        assert got[2] is dw
        R.check_head(got, x, w, tgt, 1.0, EPS, f"accumulate {dtype} {piece}", base=base)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_few_rows_without_a_target(dtype):
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    T, V, d = 7, 520, 40
    m = _model(fd, V, d, dtype)
    x, w, tgt = _case(torch, T, V, d, dtype, 6, ignore=0.0)
    tgt[0], tgt[4] = R.IGNORE, R.IGNORE
    dirty = tuple(t.clone() for t in x)
    dirty[0][0], dirty[1][4] = float("nan"), float("inf")
    got = m.head_grad(dirty, w, tgt, eps=EPS)
    torch.cuda.synchronize()
    R.check_head(got, x, w, tgt, 1.0, EPS, "few rows")
    tgt.fill_(R.IGNORE)
    loss, dx, dw = m.head_grad(dirty, w, tgt, eps=EPS)
    assert all(float(t.float().abs().max()) == 0.0 for t in (*loss, *dx, dw))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_without_a_target(dtype):
    """They may hold anything; all of them: losses and gradients are zeros."""
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    T, V, d = 70, 520, 40
    m = _model(fd, V, d, dtype)
    x, w, tgt = _case(torch, T, V, d, dtype, 6, ignore=0.0)
    tgt[3], tgt[20:40], tgt[69] = R.IGNORE, R.IGNORE, R.IGNORE
    clean = m.head_grad(x, w, tgt, eps=EPS)
    dirty = tuple(t.clone() for t in x)
    dirty[0][3], dirty[1][25], dirty[0][30, 5], dirty[1][69] = float("nan"), float("inf"), -float("inf"), float("nan")
    got = m.head_grad(dirty, w, tgt, eps=EPS)
    torch.cuda.synchronize()
    R.check_head(got, x, w, tgt, 1.0, EPS, "NaN in rows without a target")
    for a, b in zip((*got[0], *got[1], got[2]), (*clean[0], *clean[1], clean[2])):
        assert torch.equal(a, b)
    loss = m.head_loss(dirty, w, tgt)
    assert all(bool((l[20:40] == 0).all()) and bool(l.isfinite().all()) for l in loss)
    tgt.fill_(R.IGNORE)
    for piece in (0, 256):
        loss, dx, dw = m.head_grad(dirty, w, tgt, eps=EPS, piece=piece)
        assert all(float(t.float().abs().max()) == 0.0 for t in (*loss, *dx, dw))


@pytest.mark.parametrize("T", [40, 7])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_not_a_number(dtype, T):
    """A bad target or a NaN in a row shows in that row's loss and gradient, and in dw."""
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    V, d = 600, 64
    m = _model(fd, V, d, dtype)
    for kind in range(4):
        x, w, tgt = _case(torch, T, V, d, dtype, 7, ignore=0.0)
        if kind == 0:
            tgt[5] = V
        elif kind == 1:
            tgt[5] = -1
        elif kind == 2:
            x[0][5, 0] = float("nan")
        else:
            x[1][5, 3] = float("inf")
        for piece in (0, 256):
            loss, dx, dw = m.head_grad(x, w, tgt, eps=EPS, piece=piece)
            torch.cuda.synchronize()
            for t in (*loss, *dx):
                bad = ~t.isfinite().reshape(T, -1).all(1)
                assert bad.tolist() == [i == 5 for i in range(T)], kind
            assert not bool(dw.isfinite().any(1).all())
            only = m.head_loss(x, w, tgt, piece=piece)
            assert all(torch.equal(a.isfinite(), b.isfinite()) for a, b in zip(only, loss))


@pytest.mark.parametrize("T", [90, 6])
@pytest.mark.parametrize("dtype,half", [("bf16", 0.05), ("bf16", 0.3), ("bf16", 1.0), ("f32", 0.05), ("f32", 0.3), ("f32", 3.0)])
def test_points_far_apart(dtype, half, T):
    """Half differences of the logits from far below 1/16 to beyond the series (x's half difference
    alone: products of two half differences are left out)."""
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    V, d = 1200, 48
    m = _model(fd, V, d, dtype)
    x, w, tgt = _case(torch, T, V, d, dtype, 8, half=half)
    w = (w[0], torch.zeros_like(w[0]))
    ld = R.f64(x[1]) @ R.f64(w[0]).T
    say(f"largest half difference {float(ld.abs().max()):.2f}")
    for piece in (0, 512):
        got = m.head_grad(x, w, tgt, eps=1.0, piece=piece)
        torch.cuda.synchronize()
        R.check_head(got, x, w, tgt, 1.0, 1.0, f"half {half} {dtype}")


@pytest.mark.parametrize("T", [20, 8])
@pytest.mark.parametrize("dtype,reach", [("bf16", 28.0), ("f32", 290.0)])
def test_half_differences_at_the_end_of_their_range(dtype, reach, T):
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    V, d = 512, 32
    m = _model(fd, V, d, dtype)
    x, w, tgt = _case(torch, T, V, d, dtype, 9, half=1.0)
    w = (w[0], torch.zeros_like(w[0]))
    ld = R.f64(x[1]) @ R.f64(w[0]).T
    x = (x[0], (x[1].double() * (reach / float(ld.abs().max()))).to(x[1].dtype))
    loss, dx, dw = m.head_grad(x, w, tgt, eps=1.0)
    wl, wx, ww = R.head(x, w, tgt, 1.0, 1.0)
    lim = 2 * R.half_step(x[0].dtype) + 1e-5
    for a, b, tol in ((loss[0], wl[0], 1e-5), (loss[1], wl[1], 1e-5), (dx[0], wx[0], lim), (dx[1], wx[1], lim), (dw, ww, lim)):
        assert float(torch.linalg.norm(R.f64(a) - b) / torch.linalg.norm(b)) <= tol


def test_large_logits():
    """Logits of some hundreds: one column holds nearly all of a row's weight."""
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    for dtype in ("bf16", "f32"):
        T, V, d = 50, 904, 64
        m = _model(fd, V, d, dtype)
        x, w, tgt = _case(torch, T, V, d, dtype, 10, size=100.0, half=1e-6)
        got = m.head_grad(x, w, tgt, eps=EPS, piece=256)
        torch.cuda.synchronize()
        R.check_head(got, x, w, tgt, 1.0, EPS, f"large logits {dtype}")


def test_no_rows():
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    m = _model(fd, 16, 8, "bf16")
    x = tuple(torch.empty(0, 8, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    w = tuple(torch.ones(16, 8, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    tgt = torch.empty(0, dtype=torch.int32, device="cuda")
    assert m.head_loss(x, w, tgt)[0].numel() == 0
    dw = torch.ones(16, 8, dtype=torch.bfloat16, device="cuda")
    m.head_grad(x, w, tgt, dw=dw)
    assert float(dw.float().abs().max()) == 0.0
    dw = torch.ones(16, 8, device="cuda")
    m.head_grad(x, w, tgt, dw=dw, accumulate=True)
    assert bool((dw == 1).all())


@pytest.mark.parametrize("dtype,piece", [("bf16", 0), ("bf16", 131072), ("f32", 131072)])
def test_offsets_beyond_32_bits(dtype, piece):
    """More than 2^31 logits: the last rows and the last columns against the statement."""
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    T, V, d = 17000, 131072, 8
    m = _model(fd, V, d, dtype)
    x, w, tgt = _case(torch, T, V, d, dtype, 14, half=1e-2)
    loss, dx, dw = m.head_grad(x, w, tgt, eps=EPS, piece=piece)
    torch.cuda.synchronize()
    # rows are independent of each other
    rows = torch.cat([torch.arange(40), torch.arange(T - 90, T)]).cuda()
    xs, ts = tuple(t[rows] for t in x), tgt[rows]
    want, bound = R.head(xs, w, ts, 1.0, EPS), R.head_bound(xs, w, ts, 1.0, EPS)
    for a, v, b, c in zip((*loss, *dx), (*want[0], *want[1]), (*bound[0], *bound[1]), ("loss.m", "loss.d", "dx.m", "dx.d")):
        R.check(a[rows], v, b, c)
    # the gradient of w at some of its rows, from the whole batch in float64 on the device
    cols = torch.cat([torch.arange(30), torch.arange(V - 60, V)]).cuda()
    live = (tgt != R.IGNORE).double()[:, None]
    at = []
    for sign in (1.0, -1.0):
        xx, g = x[0].double() + sign * x[1].double(), torch.empty(T, len(cols), device="cuda", dtype=torch.float64)
        ww = w[0].double() + sign * w[1].double()
        for i in range(0, T, 2048):
            g[i:i + 2048] = torch.softmax(xx[i:i + 2048] @ ww.T, -1)[:, cols]
        g -= (tgt[:, None] == cols[None]).double()
        at.append((g * live).T @ xx)
    want = ((at[0] - at[1]) / (2 * EPS)).cpu()
    got = R.f64(dw[cols])
    # the product left out of the logits' mean (1e-2 of x times 1e-2 of w here) moves every probability
    # by at most as much of itself
    left = float((x[1].double() @ w[1][cols].double().T).abs().max())
    assert left < 2e-3
    assert float(torch.linalg.norm(got - want) / torch.linalg.norm(want)) <= 2 * R.half_step(x[0].dtype) + 1e-5 + left


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_graph_and_stream(dtype):
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    T, V, d = 75, 1040, 96
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        m = _model(fd, V, d, dtype, stream=st.cuda_stream)
        x, w, tgt = _case(torch, T, V, d, dtype, 11)
        scr = m.head_scratch(T, 512)
        out = m.head_grad(x, w, tgt, eps=EPS, piece=512, scratch=scr)
        st.synchronize()

        def step():
            m.head_grad(x, w, tgt, eps=EPS, piece=512, loss=out[0], dx=out[1], dw=out[2], scratch=scr)

        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            step()
        for k in range(4):
            nx, nw, nt = _case(torch, T, V, d, dtype, 20 + k)
            for a, b in ((x[0], nx[0]), (x[1], nx[1]), (w[0], nw[0]), (w[1], nw[1]), (tgt, nt)):
                a.copy_(b)
            graph.replay()
            st.synchronize()
            got = [t.clone() for t in (*out[0], *out[1], out[2])]
            R.check_head((got[:2], got[2:4], got[4]), x, w, tgt, 1.0, EPS, f"replay {k}")
            step()
            st.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, (*out[0], *out[1], out[2])))


def test_two_streams_at_once():
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    T, V, d = 300, 2048, 128
    jobs = []
    for k in range(2):
        st = torch.cuda.Stream()
        m = _model(fd, V, d, "bf16", stream=st.cuda_stream)
        jobs.append((st, m, _case(torch, T, V, d, "bf16", 30 + k), m.head_scratch(T, 512)))
    torch.cuda.synchronize()
    outs = [None, None]
    for _ in range(4):
        for k, (st, m, (x, w, tgt), scr) in enumerate(jobs):
            with torch.cuda.stream(st):
                outs[k] = m.head_grad(x, w, tgt, eps=EPS, piece=512, scratch=scr)
    torch.cuda.synchronize()
    for (_, _, (x, w, tgt), _), got in zip(jobs, outs):
        R.check_head(got, x, w, tgt, 1.0, EPS, "two streams")


def test_from_tokens_to_losses_and_back():
    """The two ends together, as a model without layers: lookup, loss, both gradients of a tied
    table added up, and the table's entries of Hv against differences of its gradient."""
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    B, S, V, d, scale = 3, 21, 200, 48, 3.5
    m = _model(fd, V, d, "f32", embed_scale=scale)
    g = torch.Generator().manual_seed(12)
    th = (torch.randn(V, d, generator=g) * 0.3).cuda()
    v = torch.randn(V, d, generator=g).cuda()
    tok = torch.randint(0, V, (B, S), generator=g).to(torch.int32).cuda()
    tgt = torch.cat([tok[:, 1:], torch.full((B, 1), R.IGNORE, dtype=torch.int32, device="cuda")], 1).reshape(-1)
    n = B * (S - 1)
    x = m.embed_forward(tok, (th, v), eps=EPS)
    hv = torch.empty(V, d, device="cuda")
    loss, dx, _ = m.head_grad(x, (th, EPS * v), tgt, scale=1.0 / n, eps=EPS, piece=256, dw=hv)
    m.embed_backward(dx[1], tok, eps=EPS, out=hv, accumulate=True)
    torch.cuda.synchronize()

    # the statement (fp32 models of this size leave nothing out)
    t, dv = R.f64(th), EPS * R.f64(v)
    tk, keep = tok.cpu().long(), tgt.cpu() != R.IGNORE
    xm, xd = (scale * a[tk].reshape(-1, d) for a in (t, dv))
    lm, ld = xm @ t.T + xd @ dv.T, xd @ t.T + xm @ dv.T
    y = tgt.cpu().long().clamp(0)
    at = [torch.softmax(l, -1) - torch.nn.functional.one_hot(y, V) for l in (lm + ld, lm - ld)]
    gm, gd = ((a * keep[:, None] / n) for a in ((at[0] + at[1]) / 2, (at[0] - at[1]) / 2))
    want = (gm.T @ xd + gd.T @ xm) / EPS
    want.index_add_(0, tk.reshape(-1), scale / EPS * (gd @ t + gm @ dv))
    assert float(torch.linalg.norm(R.f64(hv) - want) / torch.linalg.norm(want)) < 3e-6

    def grad(w):
        w = w.requires_grad_()
        lg = (scale * w[tk])[:, :-1].reshape(-1, d) @ w.T
        l = torch.nn.functional.cross_entropy(lg, tk[:, 1:].reshape(-1))
        return l.detach(), torch.autograd.grad(l, w)[0]

    # the derivative itself, of losses in fp64 (their rounding, 2^-52 of 5, over 2 eps: 1e-12)
    (lp, gp), (ln, gn) = grad(t + dv), grad(t - dv)
    diff = (gp - gn) / (2 * EPS)
    assert float(torch.linalg.norm(R.f64(hv) - diff) / torch.linalg.norm(diff)) < 3e-6
    assert abs(float(loss[0].double().sum() / n) - float(lp + ln) / 2) < 1e-6 * abs(float(lp + ln))
    assert abs(float(loss[1].double().sum() / n) - float(lp - ln) / 2) < 1e-5 * abs(float(lp - ln))


@pytest.mark.parametrize("T,V,d,pad,dtype,piece", [
    (1100, 8192, 4096, 8, "bf16", 0), (1100, 8192, 4096, 0, "bf16", 1000), (1100, 8192, 4096, 0, "bf16", 8192),
    (517, 12008, 4104, 0, "bf16", 4096), (60, 262136, 2048, 0, "f32", 65536)])
def test_large_batches_skip_rows_without_a_target(T, V, d, pad, dtype, piece):
    """Large enough that only the rows with a target are multiplied: the others may hold anything, and no row's
    result depends on which of the others have a target."""
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    m = _model(fd, V, d, dtype)
    x, w, full = _case(torch, T, V, d, dtype, 15, pad=pad, ignore=0.0)
    dt = torch.float32

    def run(x, tgt):
        dx = tuple(torch.full((T, d), 5.0, dtype=dt, device="cuda") for _ in range(2))
        got = m.head_grad(x, w, tgt, eps=EPS, piece=piece, dx=dx, dw=torch.full((V, d), 5.0, dtype=dt, device="cuda"))
        alone = m.head_loss(x, w, tgt, piece=piece)
        torch.cuda.synchronize()
        for q in (0, 1):
            R.check(alone[q], R.f64(got[0][q]), R.f64(got[0][q]).abs() * 1e-6 + 1e-6, "loss alone")
        return got

    whole = run(x, full)
    g = torch.Generator().manual_seed(16)
    t = torch.arange(T)
    masks = {"scattered": torch.rand(T, generator=g) < 0.3, "most": torch.rand(T, generator=g) < 0.9, "the end": t >= T // 3,
             "the start": t < T - 7, "all but one": t != T // 2, "all": t >= 0}
    for name, none in masks.items():
        say(f"T {T} V {V} d {d} {dtype} piece {piece} without a target: {name}")
        none = none.cuda()
        tgt = torch.where(none, torch.full_like(full, R.IGNORE), full)
        dirty = tuple(torch.where(none[:, None], torch.full_like(a, float("nan")), a) for a in x)
        loss, dx, dw = run(dirty, tgt)
        for a, b in zip((*loss, *dx), (*whole[0], *whole[1])):
            assert torch.equal(a[~none], b[~none]) and float(a[none].abs().sum()) == 0.0
        assert bool(torch.isfinite(dw).all())
        if name == "all":
            assert float(dw.abs().max()) == 0.0
        if name == "all but one":
            # dw of one row: its gradient's outer products
            r = T // 2
            one = m.head_grad(tuple(a[r:r + 1] for a in x), w, full[r:r + 1].contiguous(), eps=EPS,
                              dw=torch.empty(V, d, device="cuda"))[2]
            assert float(torch.linalg.norm(dw - one) / torch.linalg.norm(one)) <= 2 * R.half_step(x[0].dtype) + 1e-5
        if name == "scattered" and dtype == "bf16" and piece == 0:
            R.check_head((loss, dx, dw), x, w, tgt, 1.0, EPS, "scattered")


def test_large_batch_in_rows_far_apart():
    """Rows of x spread over more than 2^31 bytes: the same bits as from contiguous ones."""
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    T, V, d = 1100, 8192, 4096
    m = _model(fd, V, d, "bf16")
    x, w, tgt = _case(torch, T, V, d, "bf16", 17, ignore=0.4)
    wide = tuple(torch.empty(T, 1 << 20, dtype=torch.bfloat16, device="cuda")[:, :d].copy_(a) for a in x)
    for piece in (0, 1024):
        got, want = m.head_grad(wide, w, tgt, eps=EPS, piece=piece), m.head_grad(x, w, tgt, eps=EPS, piece=piece)
        torch.cuda.synchronize()
        for a, b in zip((*got[0], *got[1], got[2]), (*want[0], *want[1], want[2])):
            assert torch.equal(a, b)


def test_graph_of_a_large_batch_whose_targets_change():
    """Captured once; the rows that have a target are those of each replay."""
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    T, V, d = 1100, 8192, 4096
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        m = _model(fd, V, d, "bf16", stream=st.cuda_stream)
        x, w, full = _case(torch, T, V, d, "bf16", 18, ignore=0.0)
        tgt, scratch = full.clone(), m.head_scratch(T)
        dx, dw = tuple(torch.empty_like(a) for a in x), torch.empty_like(w[0])
        loss = tuple(torch.empty(T, device="cuda") for _ in range(2))
        call = lambda: m.head_grad(x, w, tgt, eps=EPS, loss=loss, dx=dx, dw=dw, scratch=scratch)
        call()
        st.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            call()
        g = torch.Generator().manual_seed(19)
        for share in (0.3, 0.0, 0.95, 1.0, 0.5):
            tgt.copy_(torch.where(torch.rand(T, generator=g).cuda() < share, torch.full_like(full, R.IGNORE), full))
            graph.replay()
            st.synchronize()
            got = [a.clone() for a in (*loss, *dx, dw)]
            for a in (*loss, *dx, dw):
                a.fill_(7.0)
            call()
            st.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, (*loss, *dx, dw)))
