"""Which way fdh_head_loss and fdh_head_grad take (fdh_testing_head_route), and sizes that reach each of them."""
import ctypes as C

NAMES = ("thin", "fused", "order", "keep", "rows", "columns", "piece", "first")

# dtype, T, V, d, piece asked for, what the route must be: both passes of every tile (the gradient's runs where the
# vocabulary is in pieces), with rests of rows, columns and width
WAYS = [
    ("f32", 17, 1032, 56, 512, dict(fused=1, keep=0, rows=32, columns=128)),
    ("f32", 17, 1032, 56, 0, dict(fused=1, keep=1, rows=32, columns=128)),
    ("f32", 77, 1032, 72, 512, dict(fused=1, keep=0, rows=64, columns=64)),
    ("f32", 300, 1032, 40, 0, dict(fused=1, keep=1, rows=64, columns=64)),
    ("f32", 300, 14008, 120, 6144, dict(fused=1, keep=0, rows=64, columns=128)),
    ("f32", 70, 14008, 40, 0, dict(fused=1, keep=1, rows=64, columns=128)),
    ("f32", 510, 20488, 56, 8192, dict(fused=1, keep=0, rows=128, columns=128)),
    ("f32", 510, 8184, 72, 0, dict(fused=1, keep=1, rows=128, columns=128)),
    ("f32", 2001, 10248, 24, 4096, dict(fused=1, keep=0, rows=256, columns=128)),
    ("f32", 1999, 4088, 40, 0, dict(fused=1, keep=1, rows=256, columns=128)),
    ("f32", 200, 1032, 328, 512, dict(fused=0, keep=0)),
    ("f32", 300, 1032, 520, 0, dict(fused=0, keep=1)),
    ("bf16", 17, 1032, 72, 512, dict(fused=1, keep=0, rows=32, columns=128)),
    ("bf16", 77, 1032, 72, 512, dict(fused=1, keep=0, rows=64, columns=64)),
    ("bf16", 300, 14008, 120, 6144, dict(fused=1, keep=0, rows=64, columns=128)),
    ("bf16", 510, 20488, 56, 8192, dict(fused=1, keep=0, rows=128, columns=128)),
    ("bf16", 2001, 10248, 24, 4096, dict(fused=1, keep=0, rows=256, columns=128)),
    ("bf16", 1999, 4088, 40, 0, dict(fused=1, keep=1, rows=256, columns=128)),
    ("f32", 8, 1032, 56, 256, dict(thin=1, keep=1, order=0)),
]

# rows put in order, fp32: the vocabulary in pieces, and whole
ORDERED = [(8400, 32000, 96, 0, dict(fused=1, order=1, keep=0, rows=256)), (8400, 32000, 96, 32000, dict(fused=1, order=1, keep=1, rows=256))]


def route(fd, m, T, piece, grads=True):
    out = (C.c_int32 * 8)()
    assert fd.lib().fdh_testing_head_route(m._h, T, piece, int(grads), out) == 0
    return dict(zip(NAMES, out))


def expect(fd, m, T, piece, want):
    got = route(fd, m, T, piece)
    assert all(got[k] == v for k, v in want.items()), (T, piece, got, want)
