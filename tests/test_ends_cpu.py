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
    assert fd.lib().fdh_embed_scratch_bytes(m._h, 2, 5, C.byref(need)) == 0 and need.value > 0
    for x in (m, g):
        assert _bwd(x, tok=C.c_void_p(0)) == INVALID and _bwd(x, B=-2) == INVALID
        assert _bwd(x, eps=0.0) == INVALID and _bwd(x, eps=float("nan")) == INVALID
        assert _bwd(x, dx=C.c_void_p(0)) == INVALID and _bwd(x, dx=_at(1, 8)) == INVALID and _bwd(x, ldd=14) == INVALID
        assert _bwd(x, he=C.c_void_p(0)) == INVALID and _bwd(x, he=_at(3, 2)) == INVALID
        assert _bwd(x, scr=C.c_void_p(0)) == WORKSPACE and _bwd(x, n=need.value - 1) == WORKSPACE
        assert _bwd(x, scr=_at(7, 8)) == WORKSPACE
        assert _bwd(x, he=_at(1)) == INVALID and _bwd(x, scr=_at(1, 16)) == INVALID and _bwd(x, scr=_at(3, 64)) == INVALID
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
        assert n.value >= last and n.value >= 16 * B * S
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
