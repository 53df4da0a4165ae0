"""The token embedding and its gradient (fdh_embed_forward, fdh_embed_backward) against the
float64 statement of tests/ends_ref.py: widths, types, one token to some hundred thousand,
strides, positions, scales, tokens outside the vocabulary, one token everywhere, NaN,
accumulation, repeated calls, graphs, other streams; and the scale inside the HVP."""
import numpy as np
import pytest

import synth
from oracle import hvp as OH
from oracle import model as M
from tests import ends_ref as R
from tests import micro, torch_ref
from tests.gpu_util import need_gpu, rel_l2, say

pytestmark = pytest.mark.gpu

EPS = 1e-3


def _model(fd, family, V, d, dtype, max_seq=64, **kw):
    return fd.Model(family, 0, d, 1, 1, 8, V, max_seq, dtype, **kw)


def _dt(torch, dtype):
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def _rows(torch, T, n, dtype, g, pad=0, scale=1.0):
    full = torch.full((T, n + pad), 7.0, dtype=dtype)
    full[:, :n] = (torch.randn(T, n, generator=g) * scale).to(dtype)
    return full.cuda()[:, :n]


def _tokens(torch, B, S, V, g, kind="zipf"):
    if kind == "one":
        t = torch.full((B, S), min(5, V - 1))
    elif kind == "uniform":
        t = torch.randint(0, V, (B, S), generator=g)
    else:
        t = (torch.rand(B, S, generator=g) ** 6 * V).long().clamp(0, V - 1)
    return t.to(torch.int32).cuda()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V,d,B,S,pad,scale,pos", [
    (8, 8, 1, 1, 0, 1.0, False), (24, 16, 1, 2, 4, 4.0, True), (256, 64, 8, 64, 0, 0.7, False), (512, 72, 3, 7, 8, 8.5, True),
    (504, 264, 5, 50, 0, 1.0, True), (1000, 520, 2, 65, 12, 22.8, False), (8192, 1032, 1, 300, 0, 32.0, True),
    (640, 2048, 70, 1, 4, 45.2, False), (40, 4104, 1, 5, 0, 64.0, True)])
def test_forward(V, d, B, S, pad, scale, pos, dtype):
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    say(f"embed forward V {V} d {d} {B}x{S} {dtype}")
    g = torch.Generator().manual_seed(V + d)
    dt = _dt(torch, dtype)
    m = _model(fd, "gpt2" if pos else "llama", V, d, dtype, max_seq=max(2, S), embed_scale=scale)
    table = (_rows(torch, V, d, dt, g), _rows(torch, V, d, torch.float32, g))
    positions = (_rows(torch, S, d, dt, g), _rows(torch, S, d, torch.float32, g)) if pos else None
    tok = _tokens(torch, B, S, V, g)
    tok.view(-1)[-1] = -1 if V % 16 else V
    for ve, vp in ((table[1], positions and positions[1]), (None, None)):
        out = tuple(torch.full((B * S, d + pad), 3.0, device="cuda") for _ in range(2))
        ps = (positions[0], vp) if pos else None
        y = m.embed_forward(tok, (table[0], ve), eps=EPS, positions=ps, out=tuple(t[:, :d] for t in out))
        torch.cuda.synchronize()
        want, bound = R.embed_forward(tok, (table[0], ve), EPS, scale, ps)
        for a, w, b, c in zip(y, want, bound, "md"):
            R.check(a, w, b, f"x.{c}")
        assert all(bool((t[:, d:] == 3.0).all()) for t in out)      # the columns beside stay as they were


@pytest.mark.parametrize("V,d,B,S,pad,kind,pos", [
    (8, 8, 1, 1, 0, "uniform", False), (24, 16, 1, 31, 4, "zipf", True), (40, 1032, 1, 2, 0, "one", False),
    (520, 264, 2, 32, 4, "uniform", True), (64, 4104, 5, 13, 0, "zipf", False), (1000, 24, 4, 64, 0, "one", True),
    (128256, 16, 1, 256, 0, "uniform", False), (1000, 24, 1, 257, 0, "zipf", True), (256, 64, 8, 64, 0, "uniform", False),
    (504, 72, 3, 11, 8, "one", True), (512, 264, 1, 32, 0, "uniform", False), (520, 264, 1, 33, 0, "one", False),
    (1000, 520, 2, 650, 12, "zipf", True), (8192, 1032, 9, 57, 0, "zipf", False), (32000, 256, 1, 8192, 0, "zipf", False),
    (128, 40, 70, 257, 0, "zipf", True), (128256, 32, 3, 5461, 0, "uniform", False), (262136, 8, 1, 70001, 0, "uniform", False),
    (16, 8, 1, 131071, 0, "one", False), (40, 16, 2, 100000, 8, "zipf", False)])
def test_backward(V, d, B, S, pad, kind, pos):
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    say(f"embed backward V {V} d {d} {B}x{S} {kind}")
    g = torch.Generator().manual_seed(V + d + S)
    scale = 8.25
    m = _model(fd, "gpt2" if pos else "llama", V, d, "bf16", max_seq=S + 3, embed_scale=scale)
    tok = _tokens(torch, B, S, V, g, kind)
    if B * S > 1:
        tok.view(-1)[0], tok.view(-1)[B * S // 2] = V, -7      # left out of the table's sums
    dx = _rows(torch, B * S, d, torch.float32, g, pad, 1e-7)
    ms = S + 3 if pos else None
    got = m.embed_backward(dx, tok, eps=EPS)
    torch.cuda.synchronize()
    want, bound = R.embed_backward(dx, tok, V, EPS, scale, ms)
    first = got if pos else (got,)
    for a, w, b, c in zip(first, want, bound, "ep"):
        R.check(a, w, b, f"hv_{c}")
    # the same bits again, and added to what is there
    again = m.embed_backward(dx, tok, eps=EPS)
    assert all(torch.equal(a, b) for a, b in zip(first, again if pos else (again,)))
    base = [_rows(torch, w.shape[0], d, torch.float32, g, 0, 1e-3) for w in want]
    acc = [b.clone() for b in base]
    m.embed_backward(dx, tok, eps=EPS, out=acc[0], out_positions=acc[1] if pos else None, accumulate=True)
    torch.cuda.synchronize()
    want, bound = R.embed_backward(dx, tok, V, EPS, scale, ms, base if pos else (base[0], None))
    for a, w, b, c in zip(acc, want, bound, "ep"):
        R.check(a, w, b, f"hv_{c} accumulated")


def test_no_tokens():
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    m = _model(fd, "gpt2", 16, 8, "f32", max_seq=4)
    tok = torch.empty((0, 3), dtype=torch.int32, device="cuda")
    e = torch.ones(16, 8, device="cuda")
    y = m.embed_forward(tok, (e, e), positions=(e, e))
    assert y[0].shape == (0, 8)
    out = [torch.full((n, 8), 2.0, device="cuda") for n in (16, 4)]
    m.embed_backward(y[1], tok, out=out[0], out_positions=out[1], accumulate=True)
    assert all(bool((o == 2.0).all()) for o in out)
    m.embed_backward(y[1], tok, out=out[0], out_positions=out[1])
    assert all(bool((o == 0.0).all()) for o in out)


def test_nan_stays_in_its_row():
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    m = _model(fd, "llama", 64, 16, "f32")
    tok = torch.arange(96, dtype=torch.int32, device="cuda").view(1, -1) % 48
    dx = torch.randn(96, 16, device="cuda")
    dx[50] = float("inf")
    dx[70, 3] = float("nan")
    want, bound = R.embed_backward(torch.where(dx.isfinite(), dx, 0.0), tok, 64, 1.0, 1.0)
    got = m.embed_backward(dx, tok)
    assert bool(torch.isinf(got[2]).all()) and bool(torch.isnan(got[22, 3]))
    keep = torch.ones(64, dtype=torch.bool)
    keep[[2, 22]] = False
    R.check(got[keep.cuda()], want[0][keep], bound[0][keep], "the other rows")


def test_offsets_beyond_32_bits():
    """A table and an output of more than 2^31 elements, rows far into both."""
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    V, d = 262136, 8200
    m = _model(fd, "llama", V, d, "bf16")
    g = torch.Generator().manual_seed(3)
    table = torch.zeros((V, d), dtype=torch.bfloat16, device="cuda")
    tok = torch.tensor([[V - 1, 0, V - 2, V - 1]], dtype=torch.int32, device="cuda")
    rows = torch.randn(3, d, generator=g).to(torch.bfloat16).cuda()
    table[[0, V - 2, V - 1]] = rows
    y = m.embed_forward(tok, (table, None))[0]
    assert torch.equal(y, rows[[2, 0, 1, 2]].float())
    del table
    dx = torch.randn(4, d, generator=g).cuda()
    hv = m.embed_backward(dx, tok)
    assert torch.equal(hv[V - 2], dx[2]) and torch.equal(hv[0], dx[1])
    assert torch.equal(hv[V - 1], (dx[0].double() + dx[3].double()).float())
    assert float(hv[1:V - 2].abs().max()) == 0.0


def test_a_batch_of_more_than_32_bits():
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    V, d, T = 24, 8200, 264000
    m = _model(fd, "gpt2", V, d, "f32", max_seq=T)
    g = torch.Generator(device="cuda").manual_seed(4)
    tok = torch.randint(0, V, (1, T), device="cuda", generator=g, dtype=torch.int32)
    tok[0, -3:] = V - 1
    dx = torch.randn(T, d, device="cuda", generator=g)
    hv, pos = m.embed_backward(dx, tok)
    assert torch.equal(pos[-5:], dx[-5:])
    cols = torch.tensor([0, 1, 4095, 8199], device="cuda")
    x = dx[:, cols].double().cpu()
    want = torch.zeros(V, 4, dtype=torch.float64).index_add_(0, tok[0].cpu().long(), x)
    size = torch.zeros(V, 4, dtype=torch.float64).index_add_(0, tok[0].cpu().long(), x.abs())
    R.check(hv[:, cols], want, 2.0 ** -52 * T * size, "hv_e")
    del hv, pos
    e = torch.randn(V, d, device="cuda", generator=g)
    y = m.embed_forward(tok, (e, None), positions=(dx, None))[0]
    R.check(y[-4:], (e[tok[0, -4:].long()].double() + dx[-4:].double()).cpu(), torch.zeros(1, dtype=torch.float64), "x.m")


def test_graph_and_stream():
    """Captured on a stream of its own and replayed over new inputs, with eager work between."""
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    V, d, B, S = 512, 136, 3, 77
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        m = _model(fd, "gpt2", V, d, "bf16", max_seq=S, embed_scale=3.0, stream=st.cuda_stream)
        g = torch.Generator().manual_seed(5)
        table = (_rows(torch, V, d, torch.bfloat16, g), _rows(torch, V, d, torch.float32, g))
        pos = (_rows(torch, S, d, torch.bfloat16, g), _rows(torch, S, d, torch.float32, g))
        tok = _tokens(torch, B, S, V, g)
        dx = _rows(torch, B * S, d, torch.float32, g)
        scr = m.embed_scratch(B, S)
        x = tuple(torch.empty(B * S, d, device="cuda") for _ in range(2))
        hv = (torch.empty(V, d, device="cuda"), torch.empty(S, d, device="cuda"))

        def step():
            m.embed_forward(tok, table, eps=EPS, positions=pos, out=x)
            m.embed_backward(dx, tok, eps=EPS, out=hv[0], out_positions=hv[1], scratch=scr)

        step()
        st.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            step()
        for k in range(4):
            tok.copy_(_tokens(torch, B, S, V, g, ["zipf", "uniform", "one", "zipf"][k]))
            dx.copy_(torch.randn(B * S, d, generator=g).cuda())
            graph.replay()
            st.synchronize()
            got = [t.clone() for t in (*x, *hv)]
            want, bound = R.embed_forward(tok, table, EPS, 3.0, pos)
            wb, bb = R.embed_backward(dx, tok, V, EPS, 3.0, S)
            for a, w, b in zip(got, [*want, *wb], [*bound, *bb]):
                R.check(a, w, b, f"replay {k}")
            step()
            st.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, (*x, *hv)))


def test_two_streams_at_once():
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    V, d, T = 4096, 512, 4000
    g = torch.Generator().manual_seed(6)
    jobs = []
    for k in range(2):
        st = torch.cuda.Stream()
        m = _model(fd, "llama", V, d, "f32", stream=st.cuda_stream)
        jobs.append((st, m, _tokens(torch, 1, T, V, g), _rows(torch, T, d, torch.float32, g), m.embed_scratch(1, T),
                     torch.empty(V, d, device="cuda")))
    torch.cuda.synchronize()
    for _ in range(5):
        for st, m, tok, dx, scr, out in jobs:
            with torch.cuda.stream(st):
                m.embed_backward(dx, tok, out=out, scratch=scr)
    torch.cuda.synchronize()
    for _, _, tok, dx, _, out in jobs:
        want, bound = R.embed_backward(dx, tok, V, 1.0, 1.0)
        R.check(out, want[0], bound[0], "hv_e")


# ---- inside the HVP --------------------------------------------------------------------
def test_scale_in_the_llama_hvp():
    """The loss at scale s is that without one at D theta, D the diagonal with s at the
    embedding, so its Hessian is D H D."""
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    f = dict(micro.MICRO["llama"], d_model=64, n_heads=4, n_kv_heads=2, d_ff=96, vocab=48, max_seq=16)
    cfg, theta, tok = micro.inputs(f, batch=3, seq=16, std=0.1)
    v = synth.rademacher_probe(4, M.num_params(cfg)).astype(np.float64)
    s = 7.5
    D = np.ones_like(theta)
    e = next(e for e in M.layout(cfg) if e.name == "embed")
    D[e.offset:e.offset + e.numel] = s
    th32 = theta.astype(np.float32)
    want = D * OH.lm_hvp(cfg, D * th32, D * v, EPS, tok)
    m = fd.Model("llama", f["n_layers"], 64, 4, 2, 96, 48, 16, "f32", embed_scale=s)
    m.set_workspace(3, 16)
    tg, vg = torch.from_numpy(th32).cuda(), torch.from_numpy(v.astype(np.float32)).cuda()
    dt = torch.from_numpy(tok).cuda()
    got = m.hvp(tg, vg, EPS, dt).cpu().numpy()
    assert rel_l2(got, want) < 1e-4
    # set on a bound operator: from the next product on
    m.set_embed_scale(1.0)
    m.bind(tg, dt, EPS)
    assert rel_l2(m.hvp_bound(vg).cpu().numpy(), OH.lm_hvp(cfg, th32, v, EPS, tok)) < 1e-4
    m.set_embed_scale(s)
    assert np.array_equal(m.hvp_bound(vg).cpu().numpy(), got)


def test_scale_in_the_gpt2_hvp():
    """GPT-2 ties its head to the embedding: only the lookup is scaled."""
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    f = dict(micro.MICRO["gpt2"], d_model=64, n_heads=4, n_kv_heads=4, d_ff=96, vocab=48, max_seq=24)
    cfg, theta, tok = micro.inputs(f, batch=3, seq=16, std=0.1)
    v = synth.rademacher_probe(4, M.num_params(cfg)).astype(np.float64)
    s, th32 = 2.5, theta.astype(np.float32)
    t = th32.astype(np.float64)
    want = (torch_ref.grad(f, t + EPS * v, tok, embed_scale=s) - torch_ref.grad(f, t - EPS * v, tok, embed_scale=s)) / (2 * EPS)
    m = fd.Model("gpt2", f["n_layers"], 64, 4, 4, 96, 48, 24, "f32", embed_scale=s)
    m.set_workspace(3, 16)
    got = m.hvp(torch.from_numpy(th32).cuda(), torch.from_numpy(v.astype(np.float32)).cuda(), EPS, torch.from_numpy(tok).cuda())
    assert rel_l2(got.cpu().numpy(), want) < 1e-4


def test_more_rows_than_one_launch_has_workgroups():
    """Four million rows and some: rows around the end of the first sweep, and the last ones."""
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    V, d, T = 64, 520, (1 << 22) + 300
    m = _model(fd, "llama", V, d, "bf16")
    g = torch.Generator().manual_seed(6)
    table, v = torch.randn(V, d, generator=g).to(torch.bfloat16).cuda(), torch.randn(V, d, generator=g).cuda()
    tok = torch.randint(0, V, (2, T // 2), generator=g, dtype=torch.int32).cuda()
    tok[0, 3] = V
    y, yd = m.embed_forward(tok, (table, v))
    flat = tok.view(-1).long()
    for r in (slice(0, 3), slice((1 << 22) - 200, T)):
        assert torch.equal(y[r], table[flat[r]].float()) and torch.equal(yd[r], v[flat[r]])
    assert bool(y[3].isnan().all()) and int(y[:, 0].isnan().sum()) == 1
