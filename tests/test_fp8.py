"""8-bit blocks without a GPU: the reference against itself, sizes, and what the entries refuse (nothing is launched)."""
import ctypes as C

import numpy as np
import pytest

import paper_2410_16926_amd as pvq
from tests import fp8_reference as ref

INVALID, UNSUPPORTED, ALIGNMENT = -1, -2, -3
# addresses that no refused call follows
A16, ODD = 0x10000, 0x10001
F32, F16, BF16 = 0, 1, 2


def test_the_reference_rounds_to_the_nearest_code():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((20, 300)) * np.exp(3 * rng.standard_normal((20, 300)))
    codes, exps = ref.encode(x)
    back = ref.decode(codes, exps, 300)
    scale = np.ldexp(1.0, np.repeat(exps[:, :3].astype(int) - 127, 128, axis=1))[:, :300]
    # half a step: 2^-4 of the value, and 2^-10 of the scale below the normal numbers
    assert (np.abs(back - x) <= np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** -10 * scale)).all()
    assert (np.abs(x) <= 448 * scale).all()
    # the scale is the least one: half of it would not do for the largest value of the block
    for b in range(3):
        part = slice(128 * b, min(300, 128 * (b + 1)))
        assert (np.abs(x[:, part]).max(axis=1) > 224 * scale[:, part.start]).all()
    again = ref.encode(back)
    assert np.array_equal(ref.decode(*again, 300), back)


def test_the_slopes_of_the_reference_are_its_differences():
    g, h = np.linspace(-9, 9, 401), 1e-5
    for name in ("silu", "gelu"):
        d = (ref.act(name, g + h)[0] - ref.act(name, g - h)[0]) / (2 * h)
        assert np.abs(d - ref.act(name, g)[1]).max() < 1e-9       # h^2 / 6 times a third derivative of at most a few, and rounding 1e-16 / h


@pytest.mark.parametrize("rows,cols", [(0, 0), (1, 1), (3, 128), (5, 129), (7, 512), (7, 513), (28672, 8192)])
def test_sizes(rows, cols):
    a, b = C.c_size_t(), C.c_size_t()
    assert pvq.lib().pvq_fp8_sizes(rows, cols, C.byref(a), C.byref(b)) == 0
    c, e = ref.planes(rows, cols)
    assert (a.value, b.value) == (rows * c, rows * e)
    assert pvq.lib().pvq_fp8_sizes(rows, cols, None, None) == 0


def test_sizes_refuse():
    L = pvq.lib()
    assert L.pvq_fp8_sizes(-1, 4, None, None) == INVALID
    assert L.pvq_fp8_sizes(4, -1, None, None) == INVALID
    assert L.pvq_fp8_sizes(1, (1 << 22) + 1, None, None) == UNSUPPORTED


def test_encode_and_decode_refuse():
    L = pvq.lib()
    for f in (lambda x, t, r, c, ld, codes, exps: L.pvq_fp8_encode(x, t, r, c, ld, codes, exps, None),
              lambda x, t, r, c, ld, codes, exps: L.pvq_fp8_decode(codes, exps, r, c, x, t, ld, None)):
        assert f(A16, F32, 0, 5, 5, None, None) == 0 and f(A16, F32, 5, 0, 0, None, None) == 0      # nothing to do
        assert f(None, F32, 2, 5, 5, A16, A16) == INVALID
        assert f(A16, F32, 2, 5, 5, None, A16) == INVALID
        assert f(A16, F32, 2, 5, 5, A16, None) == INVALID
        assert f(A16, 3, 2, 5, 5, A16, A16) == INVALID
        assert f(A16, F32, 2, 5, 4, A16, A16) == INVALID
        assert f(A16, F32, -2, 5, 5, A16, A16) == INVALID
        assert f(ODD + 1, F32, 2, 5, 5, A16, A16) == ALIGNMENT
        assert f(ODD, BF16, 2, 5, 5, A16, A16) == ALIGNMENT
        assert f(A16, F32, 2, 5, 5, A16 + 8, A16) == ALIGNMENT
        assert f(A16, F32, 2, 5, 5, A16, A16 + 2) == ALIGNMENT


def test_products_refuse():
    L = pvq.lib()

    # (a workspace that is large enough, for the shapes that want one)
    def product(m=2, n=3, k=5, a=(A16, A16), b=(A16, A16), y=A16, t=F32, ld=3):
        return L.pvq_fp8_product(*a, m, *b, n, k, y, t, ld, A16, 1 << 40, None)
    assert product(m=0) == 0 and product(n=0) == 0
    assert product(y=None) == product(ld=2) == product(t=7) == product(m=-1) == product(n=-1) == product(k=-1) == INVALID
    assert product(a=(None, A16)) == product(b=(A16, None)) == INVALID
    assert product(a=(A16 + 4, A16)) == product(b=(A16, A16 + 1)) == product(y=ODD) == ALIGNMENT
    assert product(k=(1 << 22) + 1) == UNSUPPORTED

    def dx(m=2, n=3, k=5, dy=A16, lddy=3, w=(A16, A16), out=A16, t=F32, ld=5):
        return L.pvq_fp8_input_grad(dy, lddy, m, *w, n, k, out, t, ld, A16, 1 << 40, None)
    assert dx(m=0) == 0 and dx(k=0) == 0
    assert dx(dy=None) == dx(lddy=2) == dx(ld=4) == dx(out=None) == dx(w=(A16, None)) == dx(t=-1) == dx(n=-1) == INVALID
    assert dx(dy=ODD) == dx(w=(A16 + 8, A16)) == dx(out=A16 + 2) == ALIGNMENT

    def dw(m=2, n=3, k=5, dy=A16, lddy=3, x=(A16, A16), out=A16, t=F32, ld=5):
        return L.pvq_fp8_weight_grad(dy, lddy, m, n, *x, k, out, t, ld, A16, 1 << 40, None)
    assert dw(n=0) == 0 and dw(k=0) == 0
    assert dw(dy=None) == dw(lddy=2) == dw(ld=4) == dw(out=None) == dw(x=(None, A16)) == dw(t=9) == INVALID
    assert dw(dy=ODD) == dw(x=(A16, A16 + 2)) == dw(out=A16 + 2) == ALIGNMENT


def test_the_gated_block_refuses():
    L = pvq.lib()

    def gated(m=2, n=3, k=5, act=0, h=A16, t=BF16, ld=3, hb=(None, None), kept=(None,) * 4, x=(A16, A16), g=(A16, A16), u=(A16, A16)):
        return L.pvq_fp8_gated(*x, m, *g, *u, n, k, act, h, t, ld, *hb, *kept, A16, 1 << 40, None)
    assert gated(m=0) == 0 and gated(n=0) == 0
    assert gated(act=2) == gated(t=5) == gated(ld=2) == gated(h=None) == INVALID
    assert gated(h=None, hb=(A16, None)) == gated(kept=(A16, A16, A16, None)) == gated(kept=(A16, A16, None, None)) == INVALID
    assert gated(x=(None, A16)) == gated(g=(A16, None)) == gated(u=(None, None)) == INVALID
    assert gated(hb=(A16 + 8, A16)) == gated(kept=(A16, A16, A16, A16 + 1)) == gated(h=ODD) == gated(u=(A16 + 1, A16)) == ALIGNMENT

    def backward(m=2, n=3, k=5, act=0, dh=A16, lddh=3, dx=A16, dw=(A16, A16), ldx=5, ldw=5, t=BF16, work=A16, size=1 << 30, b=(A16,) * 10):
        return L.pvq_fp8_gated_backward(dh, lddh, *b[:2], m, *b[2:6], n, k, *b[6:], act, dx, ldx, *dw, ldw, t, work, size, None)
    assert backward(k=0) == 0
    assert backward(act=-1) == backward(dh=None) == backward(lddh=2) == backward(ldx=4) == backward(ldw=4) == backward(t=3) == INVALID
    assert backward(dx=None, dw=(None, None)) == backward(dw=(A16, None)) == backward(work=None) == INVALID
    need = C.c_size_t()
    assert L.pvq_fp8_gated_backward_work_bytes(2, 3, 5, C.byref(need)) == 0 and need.value > 0
    assert backward(size=need.value - 1) == INVALID
    for i in range(10):
        assert backward(b=tuple(None if j == i else A16 for j in range(10))) == INVALID
    assert backward(work=A16 + 8) == backward(dh=ODD) == ALIGNMENT
    # workspaces: sizes, and calls whose workspace is missing, too small or not aligned
    f = L.pvq_fp8_product_work_bytes
    assert f(2, 3, 5, BF16, None) == f(2, 3, 5, 4, C.byref(need)) == f(-1, 3, 5, F32, C.byref(need)) == INVALID
    f = L.pvq_fp8_gated_work_bytes
    assert f(2, 3, 5, BF16, 0, None) == f(2, 3, 5, 4, 0, C.byref(need)) == f(2, 3, -5, F32, 0, C.byref(need)) == INVALID
    assert f(1, 28672, 8192, BF16, 0, C.byref(need)) == 0 and need.value == 0
    assert L.pvq_fp8_gated_backward_work_bytes(2, 3, 5, None) == L.pvq_fp8_gated_backward_work_bytes(2, -3, 5, C.byref(need)) == INVALID
    for f in (L.pvq_fp8_input_grad_work_bytes, L.pvq_fp8_weight_grad_work_bytes):
        assert f(A16, 8, 2, 8, 5, None) == f(A16, 8, 2, -8, 5, C.byref(need)) == INVALID
        assert f(A16, 1 << 23, 1, (1 << 22) + 1, 5, C.byref(need)) == UNSUPPORTED
        assert f(A16, 64, 2, 64, 5, C.byref(need)) == 0 and need.value == 0
        # rows that do not start at 16 bytes: small ones are taken as they are
        assert f(A16 + 2, 8, 2, 8, 5, C.byref(need)) == f(A16, 9, 2, 8, 5, C.byref(need)) == 0 and need.value == 0
        assert f(A16 + 2, 4096, 4096, 4096, 4096, C.byref(need)) == 0 and need.value >= 4096 * 4096 * 2
        assert f(A16, 4097, 4096, 4096, 4096, C.byref(need)) == 0 and need.value >= 4096 * 4096 * 2
    size = need.value
    for work, n, want in ((None, 1 << 40, INVALID), (A16, size - 1, INVALID), (A16 + 8, 1 << 40, ALIGNMENT)):
        assert L.pvq_fp8_input_grad(A16, 4097, 4096, A16, A16, 4096, 4096, A16, F32, 4096, work, n, None) == want
        assert L.pvq_fp8_weight_grad(A16, 4097, 4096, 4096, A16, A16, 4096, A16, F32, 4096, work, n, None) == want
    assert L.pvq_fp8_product_work_bytes(100, 100, 100000, BF16, C.byref(need)) == 0 and need.value > 0     # few tiles, a long sum: split
    assert L.pvq_fp8_product(A16, A16, 100, A16, A16, 100, 100000, A16, BF16, 100, None, 0, None) == INVALID
    assert L.pvq_fp8_product(A16, A16, 100, A16, A16, 100, 100000, A16, BF16, 100, A16, need.value - 1, None) == INVALID
    assert L.pvq_fp8_gated_work_bytes(100, 100, 100000, BF16, 0, C.byref(need)) == 0 and need.value > 0
    assert L.pvq_fp8_gated(A16, A16, 100, A16, A16, A16, A16, 100, 100000, 0, A16, BF16, 100, *[None] * 6, A16, need.value - 1, None) == INVALID


def test_the_binding_refuses_what_is_not_on_a_gpu():
    torch = pytest.importorskip("torch")
    x = torch.zeros(2, 128)
    planes = torch.zeros(2, 128, dtype=torch.uint8), torch.zeros(2, 4, dtype=torch.uint8)
    b = pvq.Fp8Blocks(2, 128, *planes)
    for call in (lambda: pvq.pvq_fp8_encode(x), lambda: pvq.pvq_fp8_decode(b), lambda: pvq.pvq_fp8_product(b, b),
                 lambda: pvq.pvq_fp8_input_grad(x, b), lambda: pvq.pvq_fp8_weight_grad(x, b), lambda: pvq.pvq_fp8_gated(b, b, b),
                 lambda: pvq.pvq_fp8_gated_backward(x, b, b, b, b, b)):
        with pytest.raises(ValueError):
            call()
    wide = pvq.Fp8Blocks(2, 129, *planes)
    with pytest.raises(ValueError):
        pvq.pvq_fp8_product(b, wide)
    with pytest.raises(KeyError):
        pvq.pvq_fp8_gated(b, b, b, "tanh")
    with pytest.raises(ValueError):
        pvq.pvq_fp8_gated(b, b, b, out_dtype=torch.float32, encode=True)
