"""Per-head norm and position axes of the queries and keys, without a GPU: the
configuration's checks, the layout, the oracle's gradient against autograd and
differences, and every refusal of fdh_qk_forward / fdh_qk_backward (each ends
before a launch, so addresses that nothing is behind will do)."""
import ctypes as C

import numpy as np
import pytest

import synth
from oracle import hvp as OH
from oracle import model as M

fd = pytest.importorskip("paper_2602_00816_amd.fdhvp")
torch = pytest.importorskip("torch")

from tests import qk_ref as R  # noqa: E402

HEADS = dict(d_model=48, n_heads=4, n_kv_heads=2, d_ff=40, vocab=24, max_seq=16)   # head_dim 12 in the oracle


def _create(qk, family=1, d=96, heads=4, kv=2, dtype=0):
    cfg = fd.ModelConfig(family, 1, d, heads, kv, 64, 32, 64, dtype, 1e-5, 1e4, 0, 0)
    h = C.c_void_p()
    st = fd.lib().fdh_create_qk(C.byref(cfg), None if qk is None else C.byref(qk), None, C.byref(h))
    if st == 0:
        fd.lib().fdh_destroy(h)
    else:
        assert not h.value
    return st


def _qk(norm=0, sections=(), inter=0, n=None, reserved=0):
    return fd.QkConfig(norm, len(sections) if n is None else n, (C.c_int32 * 4)(*sections), inter, reserved)


def test_create_checks_the_configuration():
    # head_dim 24: 12 rotated pairs
    for ok in (None, _qk(), _qk(1), _qk(0, (12,)), _qk(1, (4, 4, 4)), _qk(1, (4, 4, 4), 1), _qk(0, (12, 0, 0), 1),
               _qk(0, (0, 0, 0, 12)), _qk(0, (3, 3, 3, 3), 1), _qk(0, (6, 6), 1), _qk(0, (8, 2, 2), 1)):
        assert _create(ok) == 0
    for bad in (_qk(2), _qk(-1), _qk(0, (12,), 2), _qk(0, (4, 4, 4), n=5), _qk(0, (4, 4, 4), n=-1), _qk(0, (4, 4, 4), reserved=1),
                _qk(0, (4, 4, 3)), _qk(0, (4, 4, 5)), _qk(0, (14, -2)), _qk(0, (5, 7), 1), _qk(0, (2, 5, 5), 1),
                _qk(0, (2 ** 31 - 1, 13))):
        assert _create(bad) == -1
    # GPT-2 has no rotation; heads wider than 256
    assert _create(_qk(1), family=0, kv=4) == -6
    assert _create(_qk(0, (12,)), family=0, kv=4) == -6
    assert _create(_qk(), family=0, kv=4) == 0
    assert _create(_qk(1), d=4 * 264) == -6
    assert _create(None, d=4 * 264) == 0
    with pytest.raises(ValueError):
        fd.Model("llama", 1, 96, 4, 2, 64, 32, 64, rope_sections=[3, 3, 3, 2, 1])


@pytest.mark.parametrize("sections", [None, (4, 4, 4)])
def test_layout_matches_oracle(sections):
    m = fd.Model("llama", 3, 96, 4, 2, 64, 32, 64, qk_norm=True, rope_sections=sections)
    cfg = M.ModelConfig("llama", 3, 96, 4, 64, 32, 64, n_kv_heads=2, qk_norm=True, rope_sections=sections or ())
    ora, lay = M.layout(cfg), m.layout()
    assert m.num_params == M.num_params(cfg)
    for f in ("name", "offset", "numel", "layer", "kind"):
        assert [getattr(e, f) for e in lay] == [getattr(e, f) for e in ora]
    # the norm is what adds parameters, the axes add none
    assert m.num_params == fd.Model("llama", 3, 96, 4, 2, 64, 32, 64).num_params + 3 * 2 * 24
    # its workspace holds the projection before the norm, per layer (pair, fp32)
    plain = fd.Model("llama", 3, 96, 4, 2, 64, 32, 64, rope_sections=sections)
    assert m.workspace_bytes(2, 64) - plain.workspace_bytes(2, 64) >= 3 * 2 * 128 * 8 * 24 * 4


def test_models_without_heads_are_made_as_before():
    assert fd.Model("quad_diag", quad_n=10).num_params == 10
    assert fd.Model("quad_diag", n_heads=0, quad_n=10).num_params == 10
    with pytest.raises(fd.FdhError):
        fd.Model("llama", 1, 96, 0, 0, 64, 32, 64)


def test_interleaved_axes():
    cfg = M.ModelConfig("llama", 1, 96, 4, 64, 32, 64, rope_sections=(6, 4, 2), rope_interleaved=True)
    assert M.axis_of_pairs(cfg).tolist() == [0, 1, 2, 0, 1, 2, 0, 1, 0, 0, 1, 0]
    assert R.axis_of_pairs(12, (6, 4, 2), True).tolist() == M.axis_of_pairs(cfg).tolist()
    cfg.rope_interleaved = False
    assert M.axis_of_pairs(cfg).tolist() == [0] * 6 + [1] * 4 + [2] * 2
    assert R.axis_of_pairs(12, (6, 4, 2), False).tolist() == M.axis_of_pairs(cfg).tolist()


def _torch_loss(cfg, flat, tok, positions):
    """The Llama loss with the front of tests/qk_ref.py, in float64 (independent of the oracle)."""
    W = {e.name: flat[e.offset:e.offset + e.numel].view(e.shape) for e in M.layout(cfg)}
    t = torch.as_tensor(tok, dtype=torch.long)
    B, S = t.shape
    hq, hk, dh, F = cfg.n_heads, cfg.n_kv_heads, cfg.head_dim, cfg.d_ff
    ang = R.angles(dh, cfg.rope_base, B * S, S, None if positions is None else torch.as_tensor(positions),
                   cfg.rope_sections, cfg.rope_interleaved)

    def rms(x, g):
        return x / torch.sqrt((x * x).mean(-1, keepdim=True) + cfg.norm_eps) * g

    x = W["embed"][t.reshape(-1)]
    mask = torch.ones(S, S, dtype=torch.bool).triu(1)
    for l in range(cfg.n_layers):
        p = f"h{l}."
        a = rms(x, W[p + "norm1.g"])
        g = (W[p + "qnorm.g"], W[p + "knorm.g"]) if cfg.qk_norm else None
        y = R.front(a @ W[p + "wqkv"].T, hq, hk, dh, ang, g, cfg.norm_eps).view(B, S, hq + 2 * hk, dh).transpose(1, 2)
        q, k, v = y.split([hq, hk, hk], 1)
        sc = q @ k.repeat_interleave(hq // hk, 1).transpose(-1, -2) / dh ** 0.5
        o = torch.softmax(sc.masked_fill(mask, float("-inf")), -1) @ v.repeat_interleave(hq // hk, 1)
        x = x + o.transpose(1, 2).reshape(B * S, hq * dh) @ W[p + "wo"].T
        gt, up = (rms(x, W[p + "norm2.g"]) @ W[p + "wgu"].T).split([F, F], -1)
        x = x + (torch.nn.functional.silu(gt) * up) @ W[p + "wd"].T
    z = (rms(x, W["normf.g"]) @ W["head"].T).view(B, S, -1)
    return torch.nn.functional.cross_entropy(z[:, :-1].reshape(-1, cfg.vocab), t[:, 1:].reshape(-1))


@pytest.mark.parametrize("norm,sections,inter,given", [(True, (), False, False), (False, (2, 2, 2), False, True),
                                                       (True, (2, 2, 2), True, True), (True, (), False, True)])
def test_oracle_gradient_against_autograd_and_differences(norm, sections, inter, given):
    cfg = M.ModelConfig("llama", 2, qk_norm=norm, rope_sections=sections, rope_interleaved=inter, **HEADS)
    P, B, S = M.num_params(cfg), 2, 9
    theta = synth.init_params(M.init_ranges(cfg), P, 1, std=0.3).astype(np.float64)
    for e in M.layout(cfg):
        if e.kind == M.GAIN:
            theta[e.offset:e.offset + e.numel] += 0.1 * synth.normal(11, 1, e.offset, e.numel)
    tok = synth.tokens(2, B, S, cfg.vocab)
    pos = np.random.default_rng(3).integers(-50, 50, (max(1, len(sections)), B, S)) if given else None
    loss, grad = M.loss_and_grad(cfg, theta, tok, positions=pos)
    t = torch.tensor(theta, requires_grad=True)
    want = _torch_loss(cfg, t, tok, pos)
    (wg,) = torch.autograd.grad(want, t)
    assert abs(loss - float(want.detach())) <= 1e-12 * abs(loss)
    assert np.linalg.norm(grad - wg.numpy()) <= 1e-11 * np.linalg.norm(grad)
    u = synth.gaussian_direction(5, P)
    # central difference, h = 1e-4: error h^2 |L'''| / 6 against the slope
    fdiff = (M.loss(cfg, theta + 1e-4 * u, tok, positions=pos) - M.loss(cfg, theta - 1e-4 * u, tok, positions=pos)) / 2e-4
    assert abs(fdiff - grad @ u) <= 1e-6 * np.linalg.norm(grad)
    # a dataset of one batch is that batch
    a = OH.lm_hvp(cfg, theta, u, 1e-3, tok, positions=pos)
    b = OH.lm_hvp_dataset(cfg, theta, u, 1e-3, [(tok, None, pos)])
    assert np.allclose(a, b, rtol=1e-9, atol=1e-12)


# ---- refusals ----------------------------------------------------------------------
A = 1 << 40    # an aligned address that nothing dereferences


def _ctx(norm=True, dtype="bf16", axes=None, family="llama"):
    return fd.Model(family, 0, 512, 4, 2 if family == "llama" else 4, 8, 8, 64, dtype, qk_norm=norm, rope_sections=axes)


def _gains(q=A + (1 << 30), k=A + (1 << 30) + 512, vq=None, vk=None, eps=1e-3):
    return C.byref(fd.QkGains(q, k, vq, vk, eps))


def _fwd(m, g="default", pos=None, B=2, S=8, xm=A, xd=A + (1 << 20), ldx=1024, ym=A + (2 << 20), yd=A + (3 << 20), ldy=1024):
    g = _gains() if g == "default" else g
    return fd.lib().fdh_qk_forward(m._h, g, pos, B, S, xm, xd, ldx, ym, yd, ldy)


def test_forward_refusals():
    m, L = _ctx(), fd.lib()
    assert L.fdh_qk_forward(None, None, None, 1, 1, A, A, 1024, A, A, 1024) == -1
    for kw in (dict(g=None), dict(g=_gains(q=None)), dict(g=_gains(k=None)), dict(g=_gains(eps=0.0)), dict(g=_gains(eps=float("nan"))),
               dict(g=_gains(eps=-1.0)), dict(g=_gains(eps=float("inf"))), dict(B=-1), dict(S=-8), dict(xm=None), dict(xd=None),
               dict(ym=None), dict(yd=None), dict(xm=A + 8), dict(yd=A + (3 << 20) + 2), dict(ldx=1023), dict(ldx=1016),
               dict(ldy=1020), dict(ldy=1028), dict(ldx=-1024), dict(ldx=0), dict(ldy=2 ** 40),
               # overlaps: y on half of x, on the other channel of x, y_m on y_d, in place with another stride
               dict(ym=A + 2048), dict(ym=A + (1 << 20)), dict(ym=A + (3 << 20)), dict(ym=A, yd=A + (1 << 20), ldy=1032),
               dict(ym=A), dict(pos=A + (2 << 20)), dict(g=_gains(q=A + (2 << 20))), dict(g=_gains(vk=A + (3 << 20) + 64)),
               # interleaved rows whose columns do overlap (stride 2000 < 2 x 1024)
               dict(xm=A, ym=A + 2000, ldx=2000, ldy=2000)):
        assert _fwd(m, **kw) == -1, kw
        assert len(L.fdh_last_error(m._h)) > 5
    assert _fwd(m, B=1 << 20, S=1 << 12) == -6
    assert _fwd(_ctx(False)) == -1                    # gains where nothing is normed
    assert _fwd(_ctx(False, family="gpt2"), g=None) == -6
    assert fd.lib().fdh_qk_forward(fd.Model("quad_diag", quad_n=8)._h, None, None, 1, 1, A, A, 1024, A, A, 1024) == -6
    wide = fd.Model("llama", 0, 264 * 2, 2, 1, 8, 8, 64)
    assert _fwd(wide, g=None, ldx=2048, ldy=2048) == -6
    # nothing to do: no pointer is looked at
    assert _fwd(m, B=0, xm=None, ym=None) == 0
    assert _fwd(m, S=0) == 0


def _bwd(m, g="default", pos=None, B=2, S=8, xm=A, xd=A + (1 << 20), ldx=1024, gm=A + (2 << 20), gd=A + (3 << 20), lddy=1024,
         om=A + (4 << 20), od=A + (5 << 20), lddx=1024, dq=A + (6 << 20), dk=A + (7 << 20), acc=0, sc=A + (8 << 20), nb=1 << 20):
    g = _gains() if g == "default" else g
    return fd.lib().fdh_qk_backward(m._h, g, pos, B, S, xm, xd, ldx, gm, gd, lddy, om, od, lddx, dq, dk, acc, sc, nb)


def test_backward_refusals():
    m, L = _ctx(), fd.lib()
    n = C.c_size_t()
    assert L.fdh_qk_scratch_bytes(m._h, 2, 8, C.byref(n)) == 0 and n.value > 0
    for kw in (dict(g=None), dict(dq=None), dict(dk=None), dict(xm=None), dict(gm=None), dict(od=None), dict(gd=A + (3 << 20) + 4),
               dict(lddy=1022), dict(lddx=1028), dict(ldx=512), dict(om=A), dict(om=A + (2 << 20)), dict(od=A + (4 << 20) + 2048),
               dict(dq=A + (7 << 20)), dict(dq=A + (4 << 20) + 256), dict(dk=A + (2 << 20)), dict(sc=A + (4 << 20)),
               dict(sc=A + (6 << 20) - 256), dict(sc=A), dict(pos=A + (8 << 20)), dict(g=_gains(eps=0.0)), dict(B=-1)):
        assert _bwd(m, **kw) == -1, kw
    for kw in (dict(sc=None), dict(nb=n.value - 1), dict(nb=0), dict(sc=A + (8 << 20) + 8)):
        assert _bwd(m, **kw) == -2, kw
    assert _bwd(m, B=1 << 20, S=1 << 12) == -6
    plain = _ctx(False)
    assert L.fdh_qk_scratch_bytes(plain._h, 2, 8, C.byref(n)) == 0 and n.value == 0
    assert _bwd(plain, g=None) == -1                  # gain gradients where there are no gains
    assert _bwd(plain, dq=None, dk=None) == -1        # gains likewise
    assert _bwd(plain, g=None, dq=None, dk=None, om=A + (2 << 20)) == -1
    assert _bwd(plain, g=None, dq=None, dk=None, B=0) == 0
    assert L.fdh_qk_scratch_bytes(m._h, -1, 8, C.byref(n)) == -1
    assert L.fdh_qk_scratch_bytes(m._h, 1 << 20, 1 << 12, C.byref(n)) == -6
    assert L.fdh_qk_scratch_bytes(_ctx(False, family="gpt2")._h, 1, 1, C.byref(n)) == -6


def test_scratch_covers_every_smaller_batch():
    m = _ctx()
    n = C.c_size_t()
    sizes = []
    for T in list(range(0, 700)) + [4096, 4097, 5000, 16384, 1 << 20]:
        assert fd.lib().fdh_qk_scratch_bytes(m._h, 1, T, C.byref(n)) == 0
        sizes.append(n.value)
    assert sizes[0] == 0 and sizes == sorted(sizes) and sizes[-1] <= 2 * 1024 * 128 * 8


def test_bind_refuses_positions_without_a_rotation():
    L = fd.lib()
    m = fd.Model("gpt2", 1, 64, 4, 4, 64, 32, 64)
    need = C.c_size_t()
    assert L.fdh_workspace_bytes(m._h, 2, 16, 0, None, C.byref(need)) == 0
    assert L.fdh_set_workspace(m._h, C.c_void_p(A), need.value, 2, 16, 0, None) == 0
    one = (fd.Batch * 1)(fd.Batch(16, 0, 2, 16))
    pos = (C.c_void_p * 1)(C.c_void_p(A))
    assert L.fdh_bind_dataset_positions(m._h, C.c_void_p(16), one, pos, 1, 1e-3, 0, None) == -6
    assert b"positions" in L.fdh_last_error(m._h)


def test_binding_refuses_before_any_launch():
    m = _ctx(axes=(24, 20, 20))
    x = tuple(torch.zeros(4, 1024, dtype=torch.bfloat16) for _ in range(2))
    with pytest.raises(ValueError, match="device"):
        m.qk_forward(x, 4)
    with pytest.raises(ValueError, match="device"):
        m.qk_backward(tuple(t.float() for t in x), 4)
    pair = lambda x, T=4: m._qk_pair(x, "x", torch.bfloat16, T, -1)
    assert pair(x) == (x[0].data_ptr(), x[1].data_ptr(), 1024)
    for bad, word in ((tuple(t[:, :1016] for t in x), "tensors"), (tuple(t[:3] for t in x), "tensors"), ((x[0], x[1][:3]), "tensors"),
                      (tuple(t[0] for t in x), "tensors"), (tuple(t.float() for t in x), "dtype"), ((x[0], x[1].half()), "dtype"),
                      (tuple(torch.zeros(1024, 4, dtype=torch.bfloat16).T for _ in range(2)), "contiguous"),
                      ((x[0], torch.zeros(4, 1032, dtype=torch.bfloat16)[:, :1024]), "row stride")):
        with pytest.raises(ValueError, match=word):
            pair(bad)
    # one row: whatever stride torch reports for it, it is one row
    one = tuple(torch.zeros(8, 1024, dtype=torch.bfloat16)[::8] for _ in range(2))
    assert pair(one, 1)[2] == 1024


# ---- the SLQ command ----------------------------------------------------------------
def test_slq_grid_positions():
    from paper_2602_00816_amd import slq
    p = slq.grid_positions(3, 2, 13, 2, 3)
    assert p.shape == (3, 2, 13) and p.dtype == np.int32 and p.flags["C_CONTIGUOUS"]
    for s in range(13):
        assert p[:, 1, s].tolist() == [s // 6, s % 6 // 3, s % 3]
    assert slq.grid_positions(2, 1, 5, 2, 2)[:, 0].tolist() == [[0, 0, 0, 0, 1], [0, 0, 1, 1, 0]]


@pytest.mark.parametrize("args", [["--workload", "gpt2-medium-bf16", "--qk-norm"], ["--rope-sections", "24,20,21"],
                                  ["--grid", "4,4"], ["--rope-interleaved"], ["--rope-sections", "24,20,20", "--grid", "4"],
                                  ["--rope-sections", "24,20,20", "--grid", "0,4"], ["--rope-sections", "16,16,16,16"],
                                  ["--workload", "tiny-gpt2-fp32", "--rope-sections", "8"]])
def test_slq_refuses_bad_options(args, capsys):
    from paper_2602_00816_amd import slq
    with pytest.raises(SystemExit):
        slq.main(args)
    assert "error" in capsys.readouterr().err
