"""The operations that the launch timing books for the vocabulary loss: those that the kernels execute."""
import pytest

from tests import ends_points_ref as P
from tests import ends_ref as R
from tests import head_routes as H
from tests.gpu_util import need_gpu

pytestmark = pytest.mark.gpu


def _flops(torch, m, x, w, tgt, piece):
    m.timing(True)
    m.head_grad(x, w, tgt, eps=1e-2, piece=piece, dw=torch.empty(w[0].shape, device="cuda"))
    f = m.timing_read()["gemm"]["flops"]
    m.timing(False)
    return f


@pytest.mark.parametrize("dtype,T,V,d,piece", [("bf16", 17, 1032, 72, 512), ("bf16", 300, 1032, 72, 0), ("f32", 77, 1032, 72, 512),
                                               ("f32", 200, 1032, 328, 512)])
def test_every_product(dtype, T, V, d, piece):
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    m = fd.Model("llama", 0, d, 1, 1, 8, V, 2, dtype)
    x, w, tgt = P.inputs(T, V, d, dtype, 0.5, 1)
    got = _flops(torch, m, tuple(a.cuda() for a in x), tuple(a.cuda() for a in w), tgt.cuda(), piece)
    times = 1 if H.route(fd, m, T, piece)["keep"] else 2
    # four products of the logits' pair, four of dx, two of dw (over rows in whole eights)
    assert got == 2.0 * V * d * (4 * times * T + 4 * T + 2 * ((T + 7) // 8 * 8))


def test_rows_that_are_not_multiplied():
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    T, V, d = 1100, 8192, 4096
    m = fd.Model("llama", 0, d, 1, 1, 8, V, 2, "bf16")
    r = H.route(fd, m, T, 4096)
    assert r["order"] and not r["keep"]
    x, w, full = P.inputs(T, V, d, "bf16", 0.5, 1, ignore=0.0)
    x, w = tuple(a.cuda() for a in x), tuple(a.cuda() for a in w)
    for live in (T, 700, 256, 1, 0):
        tgt = torch.where(torch.arange(T) < live, full, torch.full_like(full, R.IGNORE)).cuda()
        rows = min(T, -(-live // r["rows"]) * r["rows"])
        assert _flops(torch, m, x, w, tgt, 4096) == 2.0 * V * d * (8 * rows + 4 * T + 2 * ((T + 7) // 8 * 8))


def test_hvp_in_pieces():
    """The HVP's head: three products of the logits' pair, three of dx."""
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    B, S, V, d = 2, 64, 2048, 128
    flops = []
    for piece in (0, 256):
        m = fd.Model("llama", 1, d, 2, 2, 256, V, 128, "bf16")
        m.set_vocab_piece(piece)
        m.set_workspace(B, S)
        th, v, tok = m.init_params(1), m.random_vector(3), m.make_tokens(B, S, 2)
        m.timing(True)
        m.hvp(th, v, 1e-3, tok)
        flops.append(m.timing_read()["gemm"]["flops"])
        m.timing(False)
    assert flops[1] - flops[0] == 2.0 * B * S * V * d * 3
