"""A refused bind leaves the context with the operator bound before, so the binding has to hold
on to that operator's tensors, without a GPU (stand-ins for the library and for tensors)."""
import pytest

fd = pytest.importorskip("paper_2602_00816_amd.fdhvp")
torch = pytest.importorskip("torch")


class _Tensor:
    dtype, is_cuda, shape = torch.int32, True, (2, 8)

    def __init__(self, *shape):
        self.shape = shape or self.shape

    def dim(self):
        return len(self.shape)

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 1 << 40


class _Lib:
    def __init__(self, lib, status):
        self._lib, self.status = lib, status

    def __getattr__(self, name):
        return (lambda *a: self.status) if name.startswith("fdh_bind") else getattr(self._lib, name)


@pytest.mark.parametrize("call", ["bind", "bind_dataset", "positions"])
def test_a_refused_bind_keeps_the_tensors_of_the_bound_operator(call, monkeypatch):
    m = fd.Model("llama", 1, 96, 4, 2, 64, 32, 64)
    monkeypatch.setattr(m, "_check_params", lambda p: None)
    monkeypatch.setattr(fd, "_check_tokens", lambda t: None)

    def bind(params, tok, pos):
        if call == "bind":
            m.bind(params, tok, 1e-3)
        else:
            m.bind_dataset(params, [tok], 1e-3, positions=[pos] if call == "positions" else None)

    m._L = _Lib(m._L, fd.OK)
    first = _Tensor(), _Tensor(2, 8), _Tensor(1, 2, 8)
    bind(*first)
    held = list(m._keep)
    assert all(any(t is h for h in held) for t in (first if call == "positions" else first[:2]))
    m._L.status = -1
    with pytest.raises(fd.FdhError):
        bind(_Tensor(), _Tensor(2, 8), _Tensor(1, 2, 8))
    assert len(m._keep) == len(held) and all(a is b for a, b in zip(m._keep, held))
    m._L.status = fd.OK
    second = _Tensor(), _Tensor(2, 8), _Tensor(1, 2, 8)
    bind(*second)
    assert any(t is second[0] for t in m._keep) and not any(t is first[0] for t in m._keep)
