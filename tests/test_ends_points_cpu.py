"""The bounds of tests/ends_points_ref.py, without a GPU: the pair form with every product is within
them, and without one of the two products of half differences it is not."""
import pytest

torch = pytest.importorskip("torch")

from tests import ends_points_ref as P  # noqa: E402
from tests import ends_ref as R  # noqa: E402


def _f32(got):
    return tuple(a.float() for a in got[0]), tuple(a.float() for a in got[1]), got[2].float()


@pytest.mark.parametrize("T", [8, 9, 33, 130])
@pytest.mark.parametrize("dtype,reach", [("f32", 0.5), ("f32", 1.5), ("f32", 5.0), ("bf16", 5.0), ("bf16", 28.0)])
def test_bounds_see_a_product_that_is_missing(dtype, reach, T):
    x, w, tgt = P.inputs(T, 520, 64, dtype, reach, 1)
    args = (x, w, tgt, 1.0 / T, 1e-2)
    P.check(_f32(P.statement(*args)), *args, "all products")
    for left_out in (dict(xdwd=False), dict(gdwd=False)):
        with pytest.raises(AssertionError, match="the whole|more than allowed"):
            P.check(_f32(P.statement(*args, **left_out)), *args, str(left_out))


@pytest.mark.parametrize("dtype,reach", [("f32", 290.0), ("bf16", 28.0), ("bf16", 1.5)])
def test_pair_form_is_the_two_points(dtype, reach):
    x, w, tgt = P.inputs(21, 264, 48, dtype, reach, 2)
    for a, b in zip(P.statement(x, w, tgt, 0.5, 1.0), R.head(x, w, tgt, 0.5, 1.0)):
        for p, q in zip(a, b):
            assert torch.allclose(p, q, rtol=1e-9, atol=1e-10)
