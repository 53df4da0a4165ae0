"""A scale and a step whose quotient is in range while the step's reciprocal is not."""
import pytest

from tests.gpu_util import need_gpu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [4, 40])
@pytest.mark.parametrize("scale,eps", [(0.0, 1e-310), (2e-310, 1e-310)])
def test_head_grad(T, scale, eps):
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    V, d = 264, 16
    m = fd.Model("llama", 0, d, 1, 1, 8, V, 2, "f32")
    g = torch.Generator().manual_seed(1)
    x, w = (tuple(torch.randn(n, d, generator=g).cuda() * s for s in (1.0, 1e-3)) for n in (T, V))
    tgt = torch.randint(0, V, (T,), generator=g).to(torch.int32).cuda()
    dw = m.head_grad(x, w, tgt, scale=scale, eps=eps)[2]
    want = m.head_grad(x, w, tgt, scale=2.0, eps=1.0)[2]
    # (2e-310 and 1e-310 are denormal: their quotient is 2 to 2^-46 or so)
    assert torch.allclose(dw, want * (scale / eps / 2.0), rtol=1e-6, atol=0.0)
