"""The rules of the vocabulary loss, without a GPU: the sizes that tests use for a way still reach it, and
pieces and launches cover the vocabulary within their limits."""
import itertools

import pytest

fd = pytest.importorskip("paper_2602_00816_amd.fdhvp")

from tests import head_routes as H  # noqa: E402


def _model(V, d, dtype):
    return fd.Model("llama", 0, d, 1, 1, 8, V, 2, dtype)


@pytest.mark.parametrize("dtype,T,V,d,piece,want", H.WAYS + [("f32", *o) for o in H.ORDERED])
def test_sizes_reach_their_way(dtype, T, V, d, piece, want):
    H.expect(fd, _model(V, d, dtype), T, piece, want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V,d", [(8, 8), (1000, 264), (32000, 2048), (262136, 64)])
def test_pieces(V, d, dtype):
    m = _model(V, d, dtype)
    for T, piece, grads in itertools.product((1, 8, 9, 32, 33, 500, 8192, 100003, 1 << 20), (0, 1, 300, 8192, V), (0, 1)):
        r = H.route(fd, m, T, piece, grads)
        assert r["thin"] == int(bool(grads) and T <= 8)
        assert 0 < r["piece"] <= r["first"] <= V and (r["piece"] == V or r["piece"] % 256 == 0)
        assert r["first"] == V or r["first"] % 256 == 0
        assert r["keep"] == int(bool(grads) and r["piece"] == V)
        assert T * r["first"] <= max(1 << 35, T * r["piece"]) and T * r["piece"] <= (1 << 35) + 256 * T
        assert r["fused"] or (dtype == "f32" and r["first"] == r["piece"] and not r["order"])
        if piece and not r["thin"] and T * (piece + 256) < 1 << 35:
            assert r["piece"] == min(V, (piece + 255) // 256 * 256)


def test_refusals():
    lib, m = fd.lib(), _model(64, 16, "f32")
    import ctypes as C
    out = (C.c_int32 * 8)()
    assert lib.fdh_testing_head_route(m._h, 0, 0, 1, out) == -1 and lib.fdh_testing_head_route(m._h, 1, -1, 1, out) == -1
    assert lib.fdh_testing_head_route(m._h, 1, 0, 1, None) == -1 and lib.fdh_testing_head_route(None, 1, 0, 1, out) == -1
    assert lib.fdh_testing_head_route(m._h, (1 << 20) + 1, 0, 1, out) == -6
    assert lib.fdh_testing_head_route(fd.Model("quad_diag", quad_n=4)._h, 1, 0, 1, out) == -6
