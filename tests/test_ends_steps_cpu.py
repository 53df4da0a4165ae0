"""Steps so small that dividing by them overflows, without a GPU: refused (a sum of nothing times infinity is NaN)."""
import ctypes as C

import pytest

fd = pytest.importorskip("paper_2602_00816_amd.fdhvp")

INVALID = -1
A = 1 << 40           # an address that is never followed


def _at(k):
    return C.c_void_p(A + k * (64 << 20))


@pytest.mark.parametrize("family", ["llama", "gpt2"])
@pytest.mark.parametrize("scale,eps", [(1.0, 1e-310), (1.0, 5e-324), (1e10, 1e-300), (1e-3, 1e-310)])
def test_embed_backward(family, scale, eps):
    m = fd.Model(family, 0, 16, 1, 1, 8, 64, 32, "f32", embed_scale=scale)
    hp = _at(4) if family == "gpt2" else None
    assert fd.lib().fdh_embed_backward(m._h, _at(5), 2, 5, _at(1), 16, eps, _at(3), hp, 0, _at(7), 64 << 20) == INVALID
    assert b"eps" in fd.lib().fdh_last_error(m._h)


@pytest.mark.parametrize("scale,eps", [(1.0, 1e-310), (1e-10, 1e-310), (1e30, 1e-10)])
def test_head_grad(scale, eps):
    m = fd.Model("llama", 0, 16, 1, 1, 8, 64, 32, "f32")
    inp = fd.HeadInputs(_at(1), _at(2), 16, _at(3), _at(4), _at(5), 5, 0, 0)
    g = fd.HeadGrads(_at(8), _at(9), 16, _at(10), scale, eps, 0, 0)
    assert fd.lib().fdh_head_grad(m._h, C.byref(inp), _at(6), _at(7), C.byref(g), _at(11), 64 << 20) == INVALID
