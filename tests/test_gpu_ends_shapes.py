"""Tables of the two ends whose elements are as many as they should be in another shape (w given transposed): refused
before anything is enqueued."""
import pytest

from tests.gpu_util import need_gpu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("family", ["llama", "gpt2"])
def test_tables_in_another_shape(family):
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    V, d, S = 48, 16, 32
    m = fd.Model(family, 0, d, 1, 1, 8, V, S, "f32")
    t = lambda *s: torch.zeros(*s, device="cuda")      # noqa: E731
    tok = torch.zeros(2, 3, dtype=torch.int32, device="cuda")
    x, tgt = (t(6, d), t(6, d)), tok.reshape(-1)
    good, turned = t(V, d), t(d, V)
    pos = dict(positions=(t(S, d), t(S, d))) if family == "gpt2" else {}
    calls = [lambda **k: m.embed_forward(tok, (k.get("a", good), k.get("b", good)), **pos),
             lambda **k: m.embed_backward(x[0], tok, out=k.get("a", k.get("b", good.clone()))),
             lambda **k: m.head_loss(x, (k.get("a", good), k.get("b", good)), tgt),
             lambda **k: m.head_grad(x, (k.get("a", good), good), tgt, dw=k.get("b", good.clone()))]
    for call in calls:
        call()
        for k in ("a", "b"):
            call(**{k: t(V * d)})                      # a slice of one flat vector will do
            with pytest.raises(ValueError, match="rows of 16"):
                call(**{k: turned})
    if family == "gpt2":
        for p in ((t(S, d), t(d, S)),):
            with pytest.raises(ValueError, match="rows of 16"):
                m.embed_forward(tok, (good, good), positions=p)
        with pytest.raises(ValueError, match="rows of 16"):
            m.embed_backward(x[0], tok, out_positions=t(d, S))
    torch.cuda.synchronize()
