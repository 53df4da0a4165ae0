"""The HVP with its head in pieces of the vocabulary (fdh_set_vocab_piece): against the oracle,
against whole logits, over datasets with labels, batches smaller than the plan, tied heads,
recomputation, Lanczos, and a workspace of the size that the pieces leave."""
import numpy as np
import pytest

import synth
from oracle import hvp as OH
from oracle import lanczos as OL
from oracle import model as M
from synth.workloads import WORKLOADS
from tests import micro
from tests.gpu_util import need_gpu, rel_l2, say, upload_params, workload_inputs

pytestmark = pytest.mark.gpu

EPS = 1e-3
SMALL = {
    "llama": dict(family="llama", n_layers=2, d_model=128, n_heads=4, n_kv_heads=2, d_ff=160, vocab=1000, max_seq=64, rope_base=10000.0),
    "gpt2": dict(family="gpt2", n_layers=2, d_model=128, n_heads=4, n_kv_heads=4, d_ff=160, vocab=1000, max_seq=64, rope_base=10000.0),
}


def _model(fd, f, dtype, piece, B, S, m=0, o=None, **kw):
    mod = fd.Model(f["family"], f["n_layers"], f["d_model"], f["n_heads"], f["n_kv_heads"], f["d_ff"], f["vocab"], f["max_seq"],
                   dtype, rope_base=f["rope_base"], **kw)
    mod.set_vocab_piece(piece)
    mod.set_workspace(B, S, m, o)
    return mod


@pytest.mark.parametrize("family", ["llama", "gpt2"])
@pytest.mark.parametrize("piece", [256, 512, 4096])
def test_fp32_against_the_oracle(family, piece):
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    f = SMALL[family]
    cfg, theta, tok = micro.inputs(f, batch=3, seq=40, std=0.05)
    theta = theta.astype(np.float32)
    v = synth.rademacher_probe(4, M.num_params(cfg))
    tg, vg = torch.from_numpy(theta).cuda(), torch.from_numpy(v).cuda()
    m = _model(fd, f, "f32", piece, 5, 64)
    hv = m.hvp(tg, vg, EPS, torch.from_numpy(tok).cuda())
    want = OH.lm_hvp(cfg, theta, v.astype(np.float64), EPS, tok)
    err = rel_l2(hv.cpu().numpy(), want)
    say(f"{family} piece {piece}: {err:.2e}")
    assert err < 1e-4
    whole = _model(fd, f, "f32", 0, 5, 64)
    hw = whole.hvp(tg, vg, EPS, torch.from_numpy(tok).cuda())
    assert rel_l2(hv.cpu().numpy(), hw.cpu().numpy()) < 1e-5
    for a, b in zip(m.last_losses(), whole.last_losses()):
        assert abs(a - b) < 1e-7 * abs(b)


@pytest.mark.parametrize("family", ["llama", "gpt2"])
def test_datasets_and_smaller_batches(family):
    """Labels, padding, batches of unlike sizes: the dataset average, and the bits of a batch that do
    not depend on the plan's size."""
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    f = SMALL[family]
    cfg, theta, _ = micro.inputs(f, batch=1, seq=8, std=0.05)
    theta = theta.astype(np.float32)
    v = synth.rademacher_probe(5, M.num_params(cfg))
    rng = np.random.default_rng(3)
    batches = []
    for B, S, keep in ((2, 64, 50), (5, 16, 9), (1, 8, 8)):
        tok = rng.integers(0, f["vocab"], (B, S)).astype(np.int32)
        lab = tok.copy()
        lab[:, keep:] = -100
        batches.append((tok, lab))
    tg, vg = torch.from_numpy(theta).cuda(), torch.from_numpy(v).cuda()
    dev = [tuple(torch.from_numpy(x).cuda() for x in b) for b in batches]
    want = OH.lm_hvp_dataset(cfg, theta, v.astype(np.float64), EPS, batches)
    got = []
    for plan in ((5, 64), (16, 64)):
        m = _model(fd, f, "f32", 256, *plan)
        m.bind_dataset(tg, dev, EPS)
        got.append(m.hvp_bound(vg).cpu().numpy())
    assert rel_l2(got[0], want) < 1e-4
    assert np.array_equal(got[0], got[1])
    m.set_recompute(True)
    m.set_workspace(5, 64)
    m.bind_dataset(tg, dev, EPS)
    assert np.array_equal(m.hvp_bound(vg).cpu().numpy(), got[0])


@pytest.mark.parametrize("name,layers,batch,seq,piece", [("gpt2-medium-bf16", 2, 2, 256, 8192), ("llama-1.3b-bf16", 1, 1, 384, 4096),
                                                         ("llama-1.3b-bf16", 1, 1, 384, 32000)])
def test_bf16_workload_shapes(name, layers, batch, seq, piece):
    """Against whole logits on the workloads' widths and vocabularies: both round the logits' gradient
    to bf16 (half a step: 2^-8, independently where the logits differ in their last bits)."""
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    w = dict(WORKLOADS[name], n_layers=layers)
    hv, losses = [], []
    for p in (0, piece):
        m = fd.Model.from_workload(w)
        m.set_vocab_piece(p)
        m.set_workspace(batch, seq)
        th = m.init_params(1)
        tok = m.make_tokens(batch, seq, 2, w["token_dist"])
        v = m.random_vector(3)
        hv.append(m.hvp(th, v, EPS, tok))
        losses.append(m.last_losses())
        m.close()
    err = float((hv[0] - hv[1]).double().norm() / hv[0].double().norm())
    say(f"{name} piece {piece}: {err:.2e}")
    assert err < 2 * 2.0 ** -8
    assert all(abs(a - b) < 1e-6 * abs(a) for a, b in zip(*losses))


def test_lanczos_and_workspace():
    """A run over the tiny workload agrees with the oracle's, in a workspace without logits."""
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    w = WORKLOADS["small-gpt2-fp32"]
    big = fd.Model.from_workload(w)
    whole = big.workspace_bytes(16, 512)
    big.set_vocab_piece(1024)
    assert big.workspace_bytes(16, 512) < whole - 16 * 512 * (w["vocab"] - 2048) * 16
    t = WORKLOADS["tiny-gpt2-fp32"]
    cfg, theta, tok = workload_inputs(t)
    o = fd.opts("full", 0, "f32")
    m = fd.Model.from_workload(t)
    m.set_vocab_piece(256)
    m.set_workspace(t["batch"], t["seq"], 6, o)
    th = upload_params(torch, theta, "f32")
    m.bind(th, torch.from_numpy(tok).cuda(), EPS)
    a, b, s, _ = m.lanczos(6, 3, o)
    v = synth.rademacher_probe(3, M.num_params(cfg))
    ao, bo, _ = OL.lanczos(lambda x: OH.lm_hvp(cfg, theta, x, EPS, tok), v.astype(np.float64), 6, OL.FULL)
    lg, lo = (np.linalg.eigvalsh(OL.tridiag(*x)) for x in ((a[:s], b[:s]), (ao, bo)))
    assert np.abs(lg[[0, -1]] - lo[[0, -1]]).max() < 1e-3 * np.abs(lo).max()


def test_slq_runner_with_both_ends(tmp_path):
    torch = need_gpu()
    from paper_2602_00816_amd import slq
    base = ["--workload", "tiny-gpt2-fp32", "--probes", "1", "--m", "4"]
    a = slq.main(base)
    b = slq.main(base + ["--vocab-piece", "256"])
    c = slq.main(base + ["--embed-scale", "8", "--vocab-piece", "256", "--out", str(tmp_path / "o.json")])
    assert abs(a["trace_estimate"] - b["trace_estimate"]) < 1e-3 * max(1.0, abs(a["trace_estimate"]))
    assert c["embed_scale"] == 8 and c["vocab_piece"] == 256 and c["trace_estimate"] != a["trace_estimate"]
