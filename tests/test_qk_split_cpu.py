"""How the q/k front splits its tokens and heads over wavefronts, without a GPU: everything is
covered once, nothing reaches past the scratch or the kernels' shared memory, and a launch stays
within its limits, over head counts, widths, types and lengths."""
import ctypes as C
import itertools

import pytest

fd = pytest.importorskip("paper_2602_00816_amd.fdhvp")

NAMES = ("group", "groups", "q", "k", "v", "step", "blocks", "threads", "lanes", "pairs", "rhalf", "part")
HEADS = [(1, 1), (2, 1), (3, 1), (3, 3), (4, 1), (5, 5), (6, 2), (8, 1), (16, 16), (28, 4), (32, 8), (62, 2), (128, 128), (4096, 1),
         (65536, 65536)]
TOKENS = [*range(0, 10), 15, 16, 17, 31, 33, 63, 64, 65, 129, 500, 1023, 2048, 4097, 12297, 16384, 2 ** 18 + 3, 2 ** 21 + 2 ** 12, 2 ** 31 - 64]


def _split(dtype, T, hq, hk, dh, norm, bwd, inplace=False):
    out = (C.c_int64 * 12)()
    assert fd.lib().fdh_testing_qk_split(fd.DTYPE[dtype], T, hq, hk, dh, int(norm), int(bwd), int(inplace), out) == 0
    return dict(zip(NAMES, out))


def _scratch(hq, hk, dh, dtype="f32"):
    m = fd.Model("llama", 0, hq * dh, hq, hk, 8, 8, 64, dtype, qk_norm=True)
    n = C.c_size_t()

    def at(T):
        assert fd.lib().fdh_qk_scratch_bytes(m._h, 1, T, C.byref(n)) == 0
        return n.value
    return at


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh", range(8, 257, 8))
def test_split(dh, dtype):
    half = dh // 2
    for (hq, hk), (norm, bwd, inplace) in itertools.product(HEADS, [(True, False, False), (True, True, False), (False, False, False),
                                                                    (False, False, True), (False, True, False)]):
        scratch = _scratch(hq, hk, dh, dtype) if norm and bwd else None
        for T in TOKENS:
            what = f"{hq}/{hk} heads of {dh} {dtype}, {T} tokens, norm {norm}, backward {bwd}, in place {inplace}"
            s = _split(dtype, T, hq, hk, dh, norm, bwd, inplace)
            # a head's pairs among its lanes, whole vectors of them in each half
            assert s["lanes"] in (1, 2, 4, 8, 16, 32) and half % s["pairs"] == 0, what
            assert half <= s["lanes"] * s["pairs"] < 2 * half + s["pairs"], what
            heads = 64 // s["lanes"]
            # every token in one group, every head of a group in one piece
            assert s["group"] * s["groups"] >= T and (T == 0 or s["group"] * (s["groups"] - 1) < T), what
            for H, c in ((hq, s["q"]), (hk, s["k"]), (0 if inplace else hk, s["v"])):
                assert (c - 1) * heads < s["group"] * H <= c * heads or H == c == 0, what
            pieces = s["q"] + s["k"] + s["v"]
            waves = s["blocks"] * s["threads"] // 64
            assert s["step"] <= s["groups"] and s["step"] * pieces <= waves < s["step"] * pieces + s["threads"] // 64, what
            assert (s["step"] >= 1) == (T > 0), what
            # a launch's threads; token numbers of the last group as an int
            assert s["blocks"] * s["threads"] < 2 ** 32 and s["group"] * s["groups"] < 2 ** 31, what
            # angles of the tokens that a wavefront's heads belong to, in 64 * pairs places
            tokens = 1 if s["group"] == 1 else heads
            assert tokens * half <= 64 * s["pairs"], what
            assert all(i * s["rhalf"] >> 16 == i // half for i in range(64 * s["pairs"])), what
            if scratch:
                assert 0 < s["part"] <= scratch(T) if T else s["part"] == scratch(T) == 0, what
            else:
                assert s["part"] == 0, what


def test_scratch_grows_with_the_batch():
    for hq, hk in HEADS:
        for dh in (8, 16, 40, 64, 128, 136, 256):
            at = _scratch(hq, hk, dh)
            sizes = [at(T) for T in TOKENS]
            assert sizes == sorted(sizes)


def test_split_refuses():
    out = (C.c_int64 * 12)()
    f = fd.lib().fdh_testing_qk_split
    for bad in ((2, 1, 1, 1, 8), (0, -1, 1, 1, 8), (0, 2 ** 31 - 63, 1, 1, 8), (0, 1, 0, 1, 8), (0, 1, 1, 2, 8), (0, 1, 1, 0, 8),
                (0, 1, 65537, 1, 8), (0, 1, 1, 1, 12), (0, 1, 1, 1, 264), (0, 1, 1, 1, 0)):
        assert f(*bad, 1, 1, 0, out) == -1
    assert f(0, 1, 1, 1, 8, 1, 1, 0, None) == -1
