"""The target's logits of up to 32 rows, which no rounding of a long fp32 sum reaches: a half difference whose terms
are far larger than it, in a column that weighs next to nothing, beside a mean over columns without rounding."""
import pytest

from tests import ends_ref as R
from tests.gpu_util import need_gpu, say

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [1, 2, 7, 8, 9, 31, 32])
def test_target_logits_of_few_rows(T, dtype):
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    V, d = 264, 512
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    xm, xd = torch.zeros(T, d), torch.zeros(T, d)
    wm = torch.zeros(V, d)
    tgt = (8 * torch.arange(T) + 3) % V
    xm[:, 0] = 1.0
    xd[:, 1] = 2.0 ** -6
    wm[:, 1] = 1.0                     # ld = 2^-6 in every column
    wm[tgt, 0], wm[tgt, 1] = -60.0, 0.0
    # the targets' ld: 2^12, then 28 times 2^-14 (a quarter of the half step there), then -2^12
    xd[:, 16], xd[:, 496] = 64.0, 64.0
    wm[tgt, 16], wm[tgt, 496] = 64.0, -64.0
    ks = 32 + 16 * torch.arange(28)
    xd[:, ks] = 2.0 ** -7
    for k in ks.tolist():
        wm[tgt, k] = 2.0 ** -7
    x, w = tuple(a.to(dt).cuda() for a in (xm, xd)), tuple(a.to(dt).cuda() for a in (wm, torch.zeros(V, d)))
    t = tgt.to(torch.int32).cuda()
    m = fd.Model("llama", 0, d, 1, 1, 8, V, 2, dtype)
    want = R.head(x, w, t, 1.0, 1.0)[0][1]
    assert abs(float(want[0]) - (2.0 ** -6 - 28 * 2.0 ** -14)) < 1e-15
    # the mean of 2^-6: sums of up to 264 equal terms in fp32 over another, each an exponential of 4 u
    bound = torch.full_like(want, 2 * (264 + 8) * U * 2.0 ** -6)
    for got in (m.head_loss(x, w, t)[1], m.head_loss(x, w, t, piece=256)[1], m.head_grad(x, w, t)[0][1]):
        say(f"T {T} {dtype}: off by {float((R.f64(got) - want).abs().max()):.1e}, allowed {float(bound[0]):.1e}")
        R.check(got, want, bound, f"T {T} {dtype}")
