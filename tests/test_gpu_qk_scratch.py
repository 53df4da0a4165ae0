"""The scratch of the q/k front's backward and what is summed in it: nothing is written before or
behind the bytes asked for, and the gain gradients of a batch are those of its parts."""
import pytest

from tests import qk_ref as R
from tests.gpu_util import need_gpu, say
from tests.test_gpu_qk import BASE, EPS, _dt, _gains, _model, _pair

pytestmark = pytest.mark.gpu

HEADS = [(1, 1, 8), (4, 4, 16), (5, 5, 40), (9, 3, 72), (8, 2, 128), (4, 1, 128), (3, 3, 152), (2, 1, 256)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hk,dh", HEADS)
def test_nothing_is_written_around_the_scratch(hq, hk, dh, dtype):
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    dt, ncol, room = _dt(torch, dtype), (hq + 2 * hk) * dh, 1 << 16
    m = _model(fd, hq, hk, dh, dtype)
    gains = _gains(torch, dh, dt, 1)
    for T in (1, 2, 3, 65, 700, 4099):
        say(f"{hq}/{hk} heads of {dh} {dtype}, {T} tokens")
        x = _pair(torch, T, ncol, dt, 2)
        dy = _pair(torch, T, ncol, torch.float32, 3)
        n = m.qk_scratch(1, T).numel()
        buf = torch.full((n + 2 * room,), 165, dtype=torch.uint8, device="cuda")
        dx, dg = m.qk_backward(dy, T, x=x, gains=gains, eps=EPS, scratch=buf[room:room + n])
        want, wg = m.qk_backward(dy, T, x=x, gains=gains, eps=EPS)
        assert bool((buf[:room] == 165).all()) and bool((buf[room + n:] == 165).all())
        assert all(torch.equal(a, b) for a, b in zip((*dx, *dg), (*want, *wg)))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hk,dh", HEADS)
def test_gain_gradients_are_the_sum_over_parts(hq, hk, dh, dtype):
    """The terms of a token and head have the same bits in a part and in the whole, so what
    differs are the order of the fp64 sums (as many roundings of the terms' absolute
    values as there are terms, on either side) and one rounding of every result."""
    torch = need_gpu()
    from paper_2602_00816_amd import fdhvp as fd
    T, part, ncol = 64 * 57 + 5, 64 * 7, (hq + 2 * hk) * dh
    dt = _dt(torch, dtype)
    m = _model(fd, hq, hk, dh, dtype)
    gains = _gains(torch, dh, dt, 1)
    x = _pair(torch, T, ncol, dt, 2)
    dy = _pair(torch, T, ncol, torch.float32, 3)
    pos = torch.randint(0, 5000, (1, T), dtype=torch.int32, device="cuda")
    _, whole = m.qk_backward(dy, T, x=x, gains=gains, eps=EPS, positions=pos)
    _, bound = R.backward_bound(x, dy, hq, hk, dh, R.angles(dh, BASE, T, T, pos), gains, EPS)
    sums = [torch.zeros(dh, dtype=torch.float64) for _ in range(2)]
    sizes = [torch.zeros(dh, dtype=torch.float64) for _ in range(2)]
    for a in range(0, T, part):
        b = min(T, a + part)
        _, d = m.qk_backward(tuple(t[a:b] for t in dy), b - a, x=tuple(t[a:b] for t in x), gains=gains, eps=EPS,
                             positions=pos[:, a:b].contiguous())
        for k in range(2):
            sums[k] += d[k].double().cpu()
            sizes[k] += d[k].double().cpu().abs()
    for k, H in enumerate((hq, hk)):
        terms = bound[k] / (11 * R.U32)     # the terms' absolute values, and more
        lim = 2 * T * H * 2.0 ** -53 * terms + R.U32 * (whole[k].double().cpu().abs() + sizes[k])
        assert bool(((whole[k].double().cpu() - sums[k]).abs() <= lim).all())
