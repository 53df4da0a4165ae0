"""The two ends of a model, without a GPU: every refusal of fdh_embed_* (each ends before a
launch, so addresses that nothing is behind will do), scratch sizes, and the float64
statements of tests/ends_ref.py against differences and autograd."""
import ctypes as C

import pytest

fd = pytest.importorskip("paper_2602_00816_amd.fdhvp")
torch = pytest.importorskip("torch")

from tests import ends_ref as R  # noqa: E402

INVALID, WORKSPACE, UNSUPPORTED = -1, -2, -6
A = 1 << 40           # an address that is never followed
MB = 1 << 20


def _at(k, off=0):
    return C.c_void_p(A + k * 64 * MB + off)


def _model(family="llama", V=64, d=16, dtype="f32", max_seq=32):
    return fd.Model(family, 0, d, 1, 1, 8, V, max_seq, dtype)


# ---- embedding ----------------------------------------------------------------------
def _fwd(m, tables=None, tok=None, B=2, S=5, xm=None, xd=None, ldx=16, **t):
    gpt2 = m.family == "gpt2"
    tb = dict(e=_at(1), v_e=_at(2), p=_at(3) if gpt2 else None, v_p=_at(4) if gpt2 else None, eps=1e-3)
    tb.update(t)
    w = fd.EmbedTables(tb["e"], tb["v_e"], tb["p"], tb["v_p"], tb["eps"])
    return fd.lib().fdh_embed_forward(m._h, None if tables == 0 else C.byref(w), _at(5) if tok is None else tok, B, S,
                                      _at(6) if xm is None else xm, _at(7) if xd is None else xd, ldx)


def test_embed_forward_refusals():
    m, g = _model(), _model("gpt2")
    assert _fwd(m, B=0, tok=C.c_void_p(0)) == 0 and _fwd(g, S=0) == 0      # nothing to do
    for x in (m, g):
        assert _fwd(x, tables=0) == INVALID and _fwd(x, e=None) == INVALID
        assert _fwd(x, tok=C.c_void_p(0)) == INVALID and _fwd(x, tok=_at(5, 2)) == INVALID
        assert _fwd(x, B=-1) == INVALID and _fwd(x, S=-1) == INVALID
        for eps in (0.0, -1.0, float("nan"), float("inf")):
            assert _fwd(x, eps=eps) == INVALID
        assert _fwd(x, e=_at(1, 8)) == INVALID and _fwd(x, v_e=_at(2, 2)) == INVALID
        assert _fwd(x, xm=C.c_void_p(0)) == INVALID and _fwd(x, xd=_at(7, 4)) == INVALID
        assert _fwd(x, ldx=12) == INVALID and _fwd(x, ldx=18) == INVALID and _fwd(x, ldx=(1 << 31) + 4) == INVALID
        assert _fwd(x, xd=_at(6)) == INVALID                       # one output over the other
        assert _fwd(x, xm=_at(1)) == INVALID and _fwd(x, xd=_at(2, 64)) == INVALID and _fwd(x, xm=_at(5)) == INVALID
    assert _fwd(m, p=_at(3)) == INVALID and _fwd(m, v_p=_at(4)) == INVALID
    assert _fwd(g, p=None) == INVALID and _fwd(g, p=_at(3, 4)) == INVALID and _fwd(g, S=33) == INVALID
    assert _fwd(m, B=1 << 16, S=1 << 15) == UNSUPPORTED
    assert _fwd(fd.Model("quad_diag", quad_n=10)) == UNSUPPORTED
    assert fd.lib().fdh_embed_forward(None, None, None, 1, 1, None, None, 16) == INVALID
    assert b"max_seq" in fd.lib().fdh_last_error(g._h)


def _bwd(m, tok=None, B=2, S=5, dx=None, ldd=16, eps=1e-3, he=None, hp=0, acc=0, scr=None, n=None):
    if n is None:
        n = 64 * MB
    if hp == 0:
        hp = _at(4) if m.family == "gpt2" else None
    return fd.lib().fdh_embed_backward(m._h, _at(5) if tok is None else tok, B, S, _at(1) if dx is None else dx, ldd, eps,
                                       _at(3) if he is None else he, hp, acc, _at(7) if scr is None else scr, n)


def test_embed_backward_refusals():
    m, g = _model(), _model("gpt2")
    need = C.c_size_t()
    assert fd.lib().fdh_embed_scratch_bytes(m._h, 20, 20, C.byref(need)) == 0 and need.value > 0
    for x in (m, g):
        assert _bwd(x, tok=C.c_void_p(0)) == INVALID and _bwd(x, B=-2) == INVALID
        assert _bwd(x, eps=0.0) == INVALID and _bwd(x, eps=float("nan")) == INVALID
        assert _bwd(x, dx=C.c_void_p(0)) == INVALID and _bwd(x, dx=_at(1, 8)) == INVALID and _bwd(x, ldd=14) == INVALID
        assert _bwd(x, he=C.c_void_p(0)) == INVALID and _bwd(x, he=_at(3, 2)) == INVALID
        many = dict(B=20, S=20)
        assert _bwd(x, scr=C.c_void_p(0), **many) == WORKSPACE and _bwd(x, n=need.value - 1, **many) == WORKSPACE
        assert _bwd(x, scr=_at(7, 8), **many) == WORKSPACE
        assert _bwd(x, scr=_at(1, 16), **many) == INVALID and _bwd(x, scr=_at(3, 64), **many) == INVALID
        assert _bwd(x, he=_at(1)) == INVALID and _bwd(x, he=_at(1), **many) == INVALID
        assert _bwd(x, he=_at(5, -64)) == INVALID
    assert _bwd(m, hp=_at(4)) == INVALID and _bwd(g, hp=None) == INVALID and _bwd(g, hp=_at(3, 16)) == INVALID
    assert _bwd(g, S=33) == INVALID and _bwd(m, B=1 << 16, S=1 << 15) == UNSUPPORTED
    assert _bwd(m, B=0, acc=1, scr=C.c_void_p(0), n=0, dx=C.c_void_p(0), tok=C.c_void_p(0)) == 0
    assert _bwd(fd.Model("quad_diag", quad_n=10)) == UNSUPPORTED


def test_embed_scratch_and_scale():
    lib, n = fd.lib(), C.c_size_t()
    m = _model()
    last = -1
    for B, S in ((0, 7), (1, 1), (3, 333), (1, 8192), (1, 16384), (1, 16385), (5, 100003)):
        assert lib.fdh_embed_scratch_bytes(m._h, B, S, C.byref(n)) == 0
        assert n.value >= last and n.value >= (16 * B * S if B * S > 256 else 0)
        last = n.value
    assert lib.fdh_embed_scratch_bytes(m._h, 0, 7, C.byref(n)) == 0 and n.value == 0
    assert lib.fdh_embed_scratch_bytes(m._h, -1, 7, C.byref(n)) == INVALID
    assert lib.fdh_embed_scratch_bytes(m._h, 1 << 16, 1 << 15, C.byref(n)) == UNSUPPORTED
    assert lib.fdh_embed_scratch_bytes(m._h, 1, 1, None) == INVALID
    for bad in (0.0, -1.0, float("nan"), float("inf")):
        assert lib.fdh_set_embed_scale(m._h, bad) == INVALID
        with pytest.raises(fd.FdhError):
            fd.Model("llama", 0, 16, 1, 1, 8, 64, 32, "f32", embed_scale=bad)
    assert lib.fdh_set_embed_scale(m._h, 1e-3) == 0
    assert lib.fdh_set_embed_scale(fd.Model("quad_diag", quad_n=10)._h, 2.0) == UNSUPPORTED


def test_embed_reference_is_the_gradient():
    """hv_e and hv_p are the derivatives of <dx, x> with respect to the tables, over eps."""
    g = torch.Generator().manual_seed(1)
    V, d, B, S, eps, scale = 12, 8, 2, 5, 1e-2, 3.0
    tok = torch.randint(0, V, (B, S), generator=g).to(torch.int32)
    e, p = (torch.randn(n, d, generator=g, dtype=torch.float64).requires_grad_() for n in (V, S))
    dx = torch.randn(B * S, d, generator=g, dtype=torch.float64)
    x = scale * e[tok.long()].reshape(-1, d) + p.repeat(B, 1)
    assert torch.allclose(R.embed_forward(tok, (e, None), eps, scale, (p, None))[0][0], x.detach(), rtol=1e-14)
    ge, gp = torch.autograd.grad((x * dx).sum(), (e, p))
    (he, hp), _ = R.embed_backward(dx, tok, V, eps, scale, S + 2)
    assert torch.allclose(he, ge / eps, rtol=1e-12) and torch.allclose(hp[:S], gp / eps, rtol=1e-12)
    assert float(hp[S:].abs().max()) == 0.0


# ---- loss over the vocabulary ---------------------------------------------------------
def _head(m, grads=False, T=5, ldx=16, piece=0, scr=None, n=None, loss=True, acc=0, dtype=None, scale=1.0, eps=1e-3, lddx=16,
          inputs=True, out=True, reserved=0, **at):
    p = dict(x_m=_at(1), x_d=_at(2), w_m=_at(3), w_d=_at(4), targets=_at(5), lm=_at(6), ld=_at(7), dx_m=_at(8), dx_d=_at(9), dw=_at(10))
    p.update(at)
    if not loss:
        p["lm"] = p["ld"] = None
    inp = fd.HeadInputs(p["x_m"], p["x_d"], ldx, p["w_m"], p["w_d"], p["targets"], T, piece, reserved)
    n = 64 * MB if n is None else n
    scr = _at(11) if scr is None else scr
    i = C.byref(inp) if inputs else None
    if not grads:
        return fd.lib().fdh_head_loss(m._h, i, p["lm"], p["ld"], scr, n)
    g = fd.HeadGrads(p["dx_m"], p["dx_d"], lddx, p["dw"], scale, eps, m.cfg.dtype if dtype is None else dtype, acc)
    return fd.lib().fdh_head_grad(m._h, i, p["lm"], p["ld"], C.byref(g) if out else None, scr, n)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_head_refusals(dtype):
    m = _model(dtype=dtype)
    ob = 4 if dtype == "f32" else 2
    n = C.c_size_t()
    none = C.c_void_p(0)
    for grads in (False, True):
        assert fd.lib().fdh_head_scratch_bytes(m._h, 5, 0, int(grads), C.byref(n)) == 0 and n.value > 0
        h = lambda **k: _head(m, grads, **k)      # noqa: E731
        assert h(inputs=False) == INVALID and h(T=-1) == INVALID and h(piece=-1) == INVALID and h(reserved=1) == INVALID
        assert h(T=(1 << 20) + 1) == UNSUPPORTED
        for p in ("x_m", "x_d", "w_m", "w_d"):
            assert h(**{p: none}) == INVALID and h(**{p: _at(1, 8)}) == INVALID
        assert h(targets=none) == INVALID and h(targets=_at(5, 1)) == INVALID
        assert h(ldx=8) == INVALID and h(ldx=16 + 8 // ob - 1) == INVALID and h(ldx=(1 << 20) + 8) == INVALID
        assert h(scr=none) == WORKSPACE and h(scr=_at(11, 128)) == WORKSPACE and h(n=n.value - 1) == WORKSPACE
        assert h(lm=_at(6, 2)) == INVALID and h(lm=None) == INVALID
        assert h(lm=_at(7)) == INVALID and h(lm=_at(1)) == INVALID and h(ld=_at(5, 16)) == INVALID and h(scr=_at(3)) == INVALID
        assert _head(fd.Model("quad_diag", quad_n=10), grads, dtype=0) == UNSUPPORTED
        assert _head(_model(d=(1 << 16) + 8), grads, ldx=(1 << 16) + 8, lddx=(1 << 16) + 8) == UNSUPPORTED
    assert _head(m, T=0, loss=False, scr=none, n=0, x_m=none, targets=none) == 0
    assert _head(m, loss=False) == INVALID
    g = lambda **k: _head(m, True, **k)           # noqa: E731
    assert g(out=False) == INVALID and g(dw=none) == INVALID and g(dw=_at(10, 8)) == INVALID
    assert g(dx_m=none) == INVALID and g(dx_d=_at(9, 4)) == INVALID and g(lddx=8) == INVALID and g(lddx=17) == INVALID
    for bad in (0.0, -1.0, float("nan"), float("inf")):
        assert g(eps=bad) == INVALID
    assert g(scale=float("nan")) == INVALID and g(scale=float("inf")) == INVALID
    assert g(dtype=2) == INVALID and g(dtype=-1) == INVALID
    if dtype == "f32":
        assert g(dtype=1) == INVALID
    else:
        assert g(acc=1) == INVALID                # sums of rounded gradients
    assert g(dx_d=_at(8)) == INVALID and g(dx_m=_at(1)) == INVALID and g(dw=_at(3)) == INVALID and g(dw=_at(4, 16)) == INVALID
    assert g(dw=_at(8)) == INVALID and g(scr=_at(10)) == INVALID and g(lm=_at(8), ld=_at(7)) == INVALID
    assert g(T=0, acc=1, dtype=0, scr=none, n=0, x_m=none, targets=none, dx_m=none) == 0
    assert fd.lib().fdh_head_grad(None, None, None, None, None, None, 0) == INVALID


def test_head_scratch():
    lib, n = fd.lib(), C.c_size_t()
    m = fd.Model("llama", 0, 4096, 1, 1, 8, 128256, 2, "bf16")

    def need(T, piece, grads):
        assert lib.fdh_head_scratch_bytes(m._h, T, piece, grads, C.byref(n)) == 0
        return n.value

    whole = need(16384, 128256, 1)
    assert need(16384, 0, 1) < whole / 4 and need(16384, 2048, 1) < need(16384, 0, 1)
    assert need(16384, 2048, 0) < need(16384, 2048, 1)
    assert need(16384, 2000, 1) == need(16384, 2048, 1) and need(16384, 10 ** 9, 1) == whole      # rounded up; at most the vocabulary
    assert need(0, 0, 1) == 0
    for bad in ((-1, 0, 1), (1, -1, 1)):
        assert lib.fdh_head_scratch_bytes(m._h, *bad, C.byref(n)) == INVALID
    assert lib.fdh_head_scratch_bytes(m._h, 1, 0, 1, None) == INVALID
    assert lib.fdh_head_scratch_bytes(m._h, (1 << 20) + 1, 0, 1, C.byref(n)) == UNSUPPORTED


def test_head_reference_is_the_gradient():
    g = torch.Generator().manual_seed(2)
    T, V, d, eps, scale = 9, 14, 6, 1e-2, 0.25
    x = [torch.randn(T, d, generator=g, dtype=torch.float64) * s for s in (1.0, eps)]
    w = [torch.randn(V, d, generator=g, dtype=torch.float64) * s for s in (1.0, eps)]
    tgt = torch.randint(0, V, (T,), generator=g)
    tgt[4] = R.IGNORE
    out = []
    for s in (1, -1):
        a, b = (x[0] + s * x[1]).requires_grad_(), (w[0] + s * w[1]).requires_grad_()
        l = torch.nn.functional.cross_entropy(a @ b.T, tgt, ignore_index=R.IGNORE, reduction="none")
        out.append((l.detach(), *torch.autograd.grad(scale * l.sum(), (a, b))))
    (lp, xp, wp), (lm, xm, wm) = out
    loss, dx, dw = R.head(x, w, tgt, scale, eps)
    for a, b in ((loss[0], (lp + lm) / 2), (loss[1], (lp - lm) / 2), (dx[0], (xp + xm) / 2), (dx[1], (xp - xm) / 2), (dw, (wp - wm) / (2 * eps))):
        assert torch.allclose(a, b, rtol=1e-9, atol=1e-13)


def test_vocab_piece_plan():
    """Taken at the next plan: the workspace holds pieces in place of the logits."""
    lib, need, dig = fd.lib(), C.c_size_t(), C.c_uint64()

    def total(m, B, S):
        assert lib.fdh_workspace_bytes(m._h, B, S, 0, None, C.byref(need)) == 0
        return need.value

    def digest(m):
        assert lib.fdh_testing_layout_digest(m._h, C.byref(dig)) == 0
        return dig.value

    m = fd.Model("llama", 1, 256, 2, 2, 512, 32000, 2048, "bf16")
    T = 4 * 2048
    whole = total(m, 4, 2048)
    assert lib.fdh_set_workspace(m._h, C.c_void_p(A), whole, 4, 2048, 0, None) == 0
    d0 = digest(m)
    assert lib.fdh_set_vocab_piece(m._h, 2048) == 0 and digest(m) == d0
    small = total(m, 4, 2048)
    assert whole - small > T * (32000 - 2048 - 256) * 12 - (600 << 20)
    assert total(m, 4, 2048) == small and total(m, 2, 2048) < small
    assert lib.fdh_set_workspace(m._h, C.c_void_p(A), small, 4, 2048, 0, None) == 0 and digest(m) != d0
    assert lib.fdh_set_vocab_piece(m._h, -1) == INVALID and total(m, 4, 2048) == small
    assert lib.fdh_set_vocab_piece(m._h, 0) == 0 and total(m, 4, 2048) == whole
    assert lib.fdh_set_vocab_piece(fd.Model("quad_diag", quad_n=10)._h, 256) == UNSUPPORTED


def test_ends_stay_below_the_largest_launch():
    """Sizes whose one launch would pass 2^32 threads: refused (tokens), or cut in pieces (logits)."""
    lib, n = fd.lib(), C.c_size_t()
    m = fd.Model("llama", 0, 8, 1, 1, 8, 262136, 2, "bf16")
    assert lib.fdh_embed_scratch_bytes(m._h, 1 << 14, 1 << 14, C.byref(n)) == 0
    assert lib.fdh_embed_scratch_bytes(m._h, 1, (1 << 28) + 1, C.byref(n)) == UNSUPPORTED
    T = 1 << 20
    assert lib.fdh_head_scratch_bytes(m._h, T, 262136, 0, C.byref(n)) == 0
    pieces = n.value
    assert lib.fdh_head_scratch_bytes(m._h, T, 1 << 15, 0, C.byref(n)) == 0 and n.value == pieces   # 2^35 logits
    assert lib.fdh_head_scratch_bytes(m._h, T, 1 << 14, 0, C.byref(n)) == 0 and n.value < pieces
