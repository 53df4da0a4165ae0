"""The query and key gains' entries of bf16 products, each block on its own: in the norm of a
whole product they are too few to be seen.  They are held to the 5e-2 of the bf16 parity tests;
zeros are off by 1, a wrong sign by 2, and what a lost batch makes is measured on the
oracle."""
import numpy as np
import pytest

import synth
from oracle import hvp as OH
from oracle import model as M
from tests.gpu_util import need_gpu, rel_l2, say
from tests.test_gpu_qk_hvp import EPS, SMALL, W64, W128, _cfg, _positions, _run, _theta

pytestmark = pytest.mark.gpu

TOL = 5e-2


def _gain_blocks(cfg):
    return [e for e in M.layout(cfg) if e.name.endswith(("qnorm.g", "knorm.g"))]


def _errors(cfg, got, want):
    return {e.name: rel_l2(got[e.offset:e.offset + e.numel], want[e.offset:e.offset + e.numel]) for e in _gain_blocks(cfg)}


@pytest.mark.parametrize("shape,B,S,unfused", [(SMALL, 2, 40, False), (W64, 1, 128, False), (W64, 1, 128, True), (W128, 2, 72, False),
                                               (W128, 1, 256, True)])
@pytest.mark.parametrize("axes", [False, True])
def test_gains_of_one_batch(shape, B, S, unfused, axes):
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    half = shape["d_model"] // shape["n_heads"] // 2
    w = dict(shape, dtype="bf16", qk_norm=True, rope_sections=(half - 2 * (half // 4), half // 4, half // 4) if axes else None)
    cfg = _cfg(w)
    theta = _theta(cfg)
    tok = synth.tokens(2, B, S, w["vocab"], "zipf")
    pos = _positions(3, B, S) if axes else None
    v = synth.gaussian_direction(4, theta.size).astype(np.float32)
    got, _, _, _ = _run(torch, fd, w, theta, [(tok, None, pos)], v, unfused)
    err = _errors(cfg, got, OH.lm_hvp(cfg, theta, v.astype(np.float64), EPS, tok, positions=pos))
    say(" ".join(f"{k} {e:.2e}" for k, e in err.items()))
    assert len(err) == 2 * w["n_layers"] and max(err.values()) <= TOL


@pytest.mark.parametrize("recompute", [False, True])
def test_gains_add_up_over_batches(recompute):
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    w = dict(SMALL, dtype="bf16", qk_norm=True, rope_sections=(4, 2, 2))
    cfg = _cfg(w)
    theta = _theta(cfg)
    t1, t2, t3 = (synth.tokens(30 + i, B, S, w["vocab"], "zipf") for i, (B, S) in enumerate([(2, 40), (1, 24), (3, 16)]))
    l1 = t1.copy()
    l1[0, :9] = M.IGNORE
    batches = [(t1, l1, _positions(3, 2, 40)), (t2, None, None), (t3, None, _positions(3, 3, 16, 5))]
    v = synth.gaussian_direction(4, theta.size).astype(np.float32)
    got, _, _, _ = _run(torch, fd, w, theta, batches, v, recompute=recompute)
    want = OH.lm_hvp_dataset(cfg, theta, v.astype(np.float64), EPS, batches)
    err = _errors(cfg, got, want)
    say(" ".join(f"{k} {e:.2e}" for k, e in err.items()))
    assert len(err) == 2 * w["n_layers"] and max(err.values()) <= TOL
    # a product that kept the last batch alone, or lost any one of them, is far outside
    n = [M.num_targets(t, l) for t, l, _ in batches]
    share = [OH.lm_hvp_dataset(cfg, theta, v.astype(np.float64), EPS, [b]) * k / sum(n) for b, k in zip(batches, n)]
    for lost in (share[2], want - share[0], want - share[1], want - share[2]):
        assert min(_errors(cfg, lost, want).values()) > 2 * TOL
