"""8-bit blocks on the GPU against their definition in 64 bits (tests/fp8_reference.py).

Tolerances.  h(t) = eps / 2 of a type is half a step relative to a value.
  - Codes, exponents and decoded values are exact (float16: one rounding).
  - Sums on the bfloat16 matrix instructions: products of decoded values (bfloat16 times bfloat16) are exact in float32, and K of
    them are added with an error of at most 2^-23 of a partial sum each (rounding or cutting), so
    |error| <= (K + 2) 2^-23 S, S the sum of the magnitudes.
  - Sums on the 8-bit instructions drop of each product what lies more than 13 bits below the exponent of the largest of its
    group of eight, at most 2^-13 of that one: 8 * 2^-13 of each group's largest, so |error| <= (2^-10 + (K + 2) 2^-23) S.
  - The output's rounding adds h |y|.
Where the terms are random the errors are too: in the 2-norm a K-term float32 sum is off by less than sqrt(K) 2^-23 of
sqrt(sum of squares), an 8-bit group by less than 2^-13 max / sqrt(3) a term, 2e-4 of sqrt(sum of squares) for Gaussian
terms of which the largest of eight is at most 2.9 standard deviations on average and ten times that in loud columns."""
import numpy as np
import pytest

import paper_2410_16926_amd as pvq
import synth_inputs as si
from tests import fp8_reference as ref
from tests import gpu_util as gu

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
HALF = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def blocks(c, e, cols):
    return pvq.Fp8Blocks(c.shape[0], cols, dev(c), dev(e))


def f64(t):
    return t.double().cpu().numpy()


def matrix(x, dtype, gap=0, shift=0):
    """x on the GPU in rows of cols + gap elements, starting `shift` elements behind an aligned address."""
    rows, cols = x.shape
    flat = torch.full((rows * (cols + gap) + shift + 8,), float("nan"), dtype=DTYPES[dtype], device="cuda")
    m = flat[shift:shift + rows * (cols + gap)].view(rows, cols + gap)[:, :cols]
    m.copy_(torch.from_numpy(x))
    return m


def check_blocks(b, want):
    assert ref.same_codes(b.codes.cpu().numpy(), want[0])
    assert np.array_equal(b.exponents.cpu().numpy(), want[1])


SHAPES = [(1, 1), (1, 127), (3, 128), (5, 129), (2, 1000), (17, 513), (64, 512), (33, 2049), (1, 8192), (300, 7)]


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("gap,shift", [(0, 0), (8, 0), (3, 1)])
def test_encode_and_decode(rows, cols, dtype, gap, shift):
    rng = np.random.default_rng(rows * 1000 + cols)
    x = matrix(rng.standard_normal((rows, cols)) * np.exp(2 * rng.standard_normal((rows, 1))), dtype, gap, shift)
    b = pvq.pvq_fp8_encode(x)
    want = ref.encode(f64(x))
    check_blocks(b, want)
    value = ref.decode(*want, cols)
    for t in DTYPES:
        out = matrix(np.zeros((rows, cols)), t, gap, shift)
        got = pvq.pvq_fp8_decode(b, out=out)
        assert got.data_ptr() == out.data_ptr()
        with np.errstate(over="ignore"):
            assert np.array_equal(f64(got), value.astype(np.float16).astype(np.float64) if t == "f16" else value)
        if gap:                                             # what lies between the rows stays as it was
            assert torch.isnan(torch.as_strided(out, (rows, gap), (cols + gap, 1), shift + cols)[:-1]).all()


def test_encode_of_unusual_values():
    big, tiny = np.finfo(np.float32).max, 2.0 ** -149
    rows = [np.zeros(128), -np.zeros(128), np.full(128, big), np.full(128, tiny), np.full(128, 2.0 ** -126), np.full(128, 448 * 2.0 ** -110),
            np.full(128, 448 * 2.0 ** -111), np.full(128, np.nan), np.full(128, np.inf)]
    for k in (-100, -3, 0, 7, 100):
        for top in (448.0, np.nextafter(np.float32(448), np.float32(449)), 447.999, 256.0, 255.0, 225.0, 224.0):
            row = np.linspace(-1, 1, 128) * 3
            row[17] = -top
            rows.append(row * 2.0 ** k)
    mixed = np.linspace(-5, 5, 128)
    mixed[3], mixed[70], mixed[127] = np.inf, np.nan, -np.inf
    rows.append(mixed)
    ties = (np.arange(128) + 0.5) * 2.0 ** -9                # half way between codes below 2^-6, and between others
    ties[0] = 448
    rows += [ties, -ties, ties * 64]
    x = np.array(rows).astype(np.float32)
    b = pvq.pvq_fp8_encode(dev(x))
    want = ref.encode(x.astype(np.float64))
    check_blocks(b, want)
    assert (b.exponents[:, 0].cpu().numpy() >= 17).all() and (b.exponents[:, 0].cpu().numpy() <= 247).all()
    got = f64(pvq.pvq_fp8_decode(b, torch.float32))
    value = ref.decode(*want, 128)
    value[np.abs(value) >= 2.0 ** 128] *= np.inf             # (the largest float32 rounds up out of the type)
    assert np.array_equal(got, value, equal_nan=True)


def test_decode_of_every_code_at_every_exponent():
    codes = np.tile(np.arange(256, dtype=np.uint8), (231, 1))
    exps = np.zeros((231, 4), np.uint8)
    exps[:, 0] = exps[:, 1] = np.arange(17, 248)
    b = blocks(codes, exps, 256)
    value = ref.decode(codes, exps, 256)
    value[np.abs(value) >= 2.0 ** 128] *= np.inf
    for t in ("f32", "bf16"):
        assert np.array_equal(f64(pvq.pvq_fp8_decode(b, DTYPES[t])), value, equal_nan=True)


def test_empty_matrices():
    for rows, cols in ((0, 5), (4, 0), (0, 0)):
        b = pvq.pvq_fp8_encode(torch.zeros(rows, cols, device="cuda"))
        assert pvq.pvq_fp8_decode(b, torch.bfloat16).shape == (rows, cols)
    some, none = pvq.pvq_fp8_encode(torch.ones(3, 0, device="cuda")), pvq.pvq_fp8_encode(torch.ones(2, 0, device="cuda"))
    assert torch.equal(pvq.pvq_fp8_product(some, none), torch.zeros(3, 2, device="cuda"))
    assert torch.equal(pvq.pvq_fp8_gated(some, none, none, out_dtype=torch.bfloat16), torch.zeros(3, 2, device="cuda", dtype=torch.bfloat16))
    h, g, u = pvq.pvq_fp8_gated(some, none, none, keep=True)
    assert not g.codes.any() and not u.codes.any() and not h.any()
    a = pvq.pvq_fp8_encode(torch.ones(3, 5, device="cuda"))
    dy = torch.ones(3, 0, dtype=torch.bfloat16, device="cuda")
    zero_rows = pvq.pvq_fp8_encode(torch.ones(0, 5, device="cuda"))
    assert torch.equal(pvq.pvq_fp8_input_grad(dy, zero_rows), torch.zeros(3, 5, device="cuda"))
    assert torch.equal(pvq.pvq_fp8_weight_grad(torch.ones(0, 4, dtype=torch.bfloat16, device="cuda"), zero_rows), torch.zeros(4, 5, device="cuda"))
    assert pvq.pvq_fp8_weight_grad(dy, a).shape == (0, 5)
    empty = pvq.pvq_fp8_encode(torch.ones(0, 0, device="cuda").reshape(0, 0))
    del empty
    none_kept = pvq.pvq_fp8_encode(torch.ones(0, 4, device="cuda"))
    w = pvq.pvq_fp8_encode(torch.ones(4, 5, device="cuda"))
    dx, dg, du = pvq.pvq_fp8_gated_backward(torch.ones(0, 4, dtype=torch.bfloat16, device="cuda"), zero_rows, w, w, none_kept, none_kept)
    assert dx.shape == (0, 5) and not dg.any() and not du.any() and dg.shape == (4, 5)


def check_sum(got, y, size, K, dtype, eight_bit, root):
    """got against the sum y of K terms whose magnitudes add up to `size` and whose squares to root ** 2."""
    got = f64(got)
    sums = ((2.0 ** -10 if eight_bit else 0.0) + (K + 2) * 2.0 ** -23) * size
    assert (np.abs(got - y) <= sums + HALF[dtype] * np.abs(y) + 2.0 ** -24).all(), np.abs(got - y).max()
    norm = (2e-4 if eight_bit else 0.0) * 2 + np.sqrt(K) * 2.0 ** -23 + HALF[dtype]
    assert np.linalg.norm(got - y) <= norm * np.linalg.norm(root) + 2.0 ** -24 * np.sqrt(y.size)


PRODUCTS = [(1, 1, 1), (1, 16, 128), (1, 1000, 513), (2, 17, 127), (5, 300, 1024), (16, 64, 2000), (17, 33, 129), (31, 100, 640),
            (64, 129, 256), (65, 129, 385), (100, 1000, 130), (128, 128, 1280), (129, 127, 1111), (300, 517, 900), (257, 513, 4096),
            (1000, 1, 300), (70, 3, 5000)]


@pytest.mark.parametrize("m,n,k", PRODUCTS)
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_product(m, n, k, dtype):
    rng = np.random.default_rng(m + 100 * n + 10000 * k)
    ac, ae, a = ref.random_blocks(rng, m, k)
    bc, be, b = ref.random_blocks(rng, n, k, k ** -0.5)
    y, size, root = a @ b.T, np.abs(a) @ np.abs(b).T, np.sqrt((a * a) @ (b * b).T)
    A, B = blocks(ac, ae, k), blocks(bc, be, k)
    got = pvq.pvq_fp8_product(A, B, DTYPES[dtype])
    check_sum(got, y, size, k, dtype, dtype != "f32" and m > 32, root)
    assert torch.equal(got, pvq.pvq_fp8_product(A, B, DTYPES[dtype]))
    # rows that start anywhere, and what lies between them
    out = matrix(np.zeros((m, n)), dtype, 3, 1)
    assert torch.equal(pvq.pvq_fp8_product(A, B, out=out), got)
    if m > 1:
        assert torch.isnan(torch.as_strided(out, (m - 1, 3), (n + 3, 1), 1 + n)).all()


def test_a_product_of_nan_and_of_wide_scales():
    rng = np.random.default_rng(5)
    for m in (3, 70):
        ac, ae, a = ref.random_blocks(rng, m, 300)
        bc, be, b = ref.random_blocks(rng, 40, 300)
        ac[1, 200] = 127
        for t in DTYPES:
            got = f64(pvq.pvq_fp8_product(blocks(ac, ae, 300), blocks(bc, be, 300), DTYPES[t]))
            assert np.isnan(got[1]).all() and np.isfinite(np.delete(got, 1, 0)).all()
        ac[1, 200] = 0
        ae[0], ae[2], be[5] = 17, 200, 60                     # 2^-110, 2^73 and 2^-67
        a, b = ref.decode(ac, ae, 300), ref.decode(bc, be, 300)
        y, size, root = a @ b.T, np.abs(a) @ np.abs(b).T, np.sqrt((a * a) @ (b * b).T)
        check_sum(pvq.pvq_fp8_product(blocks(ac, ae, 300), blocks(bc, be, 300), torch.float32), y, size, 300, "f32", False, root)
        check_sum(pvq.pvq_fp8_product(blocks(ac, ae, 300), blocks(bc, be, 300), torch.bfloat16), y, size, 300, "bf16", m > 32, root)


GRADS = [(1, 1, 1), (1, 64, 128), (3, 1, 129), (17, 130, 65), (64, 64, 256), (100, 257, 300), (129, 70, 1000), (517, 111, 200), (300, 513, 385), (2000, 3, 5),
         (40, 2000, 130)]


@pytest.mark.parametrize("m,n,k", GRADS)
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("gap,shift", [(0, 0), (5, 1), (8, 0)])
def test_gradients_of_a_product(m, n, k, dtype, gap, shift):
    rng = np.random.default_rng(m + 100 * n + 10000 * k)
    xc, xe, x = ref.random_blocks(rng, m, k)
    wc, we, w = ref.random_blocks(rng, n, k, k ** -0.5)
    dy_t = matrix(rng.standard_normal((m, n)), "bf16", gap, shift)
    dy = f64(dy_t)
    X, W = blocks(xc, xe, k), blocks(wc, we, k)
    for f, other, y, size, root, K, rows in (
            (pvq.pvq_fp8_input_grad, W, dy @ w, np.abs(dy) @ np.abs(w), np.sqrt((dy * dy) @ (w * w)), n, m),
            (pvq.pvq_fp8_weight_grad, X, dy.T @ x, np.abs(dy).T @ np.abs(x), np.sqrt((dy * dy).T @ (x * x)), m, n)):
        got = f(dy_t, other, DTYPES[dtype])
        check_sum(got, y, size, K, dtype, False, root)
        out = matrix(np.zeros(got.shape), dtype, gap, shift)
        assert torch.equal(f(dy_t, other, out=out), got)
        if gap and rows > 1:
            assert torch.isnan(torch.as_strided(out, (rows - 1, gap), (k + gap, 1), shift + k)).all()


def test_gradients_take_nothing_from_behind_a_row_of_dy():
    # infinities in the gap of dY's rows, and behind the last row
    rng = np.random.default_rng(9)
    m, n, k = 70, 33, 200
    xc, xe, x = ref.random_blocks(rng, m, k)
    wc, we, w = ref.random_blocks(rng, n, k)
    flat = torch.full((m + 3, n + 7), float("inf"), dtype=torch.bfloat16, device="cuda")
    flat[:m, :n] = torch.from_numpy(rng.standard_normal((m, n)))
    dy = flat[:m, :n]
    assert torch.isfinite(pvq.pvq_fp8_input_grad(dy, blocks(wc, we, k))).all()
    assert torch.isfinite(pvq.pvq_fp8_weight_grad(dy, blocks(xc, xe, k))).all()


GATED = [(1, 1, 1), (1, 130, 128), (3, 300, 513), (16, 64, 256), (33, 100, 129), (64, 257, 300), (70, 129, 385), (129, 512, 640), (300, 700, 200)]


def gated_reference(x, g, u, act):
    G, U = x @ g.T, x @ u.T
    return G, U, ref.act(act, G)[0] * U


@pytest.mark.parametrize("m,n,k", GATED)
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_gated(m, n, k, act):
    rng = np.random.default_rng(m + 100 * n + 10000 * k)
    xc, xe, x = ref.random_blocks(rng, m, k)
    gc, ge, g = ref.random_blocks(rng, n, k, k ** -0.5)
    uc, ue, u = ref.random_blocks(rng, n, k, k ** -0.5)
    X, GATE, UP = blocks(xc, xe, k), blocks(gc, ge, k), blocks(uc, ue, k)
    G, U, H = gated_reference(x, g, u, act)
    # errors of G and U as of a product; |act'| <= 1.13 and |act(g)| <= |g|, and the activation itself: its argument by a few
    # roundings relative to itself, |x| 2^-22 in the exponent and four more, times g sigma <= |g|
    S = [np.abs(x) @ np.abs(w).T for w in (g, u)]
    hats = {}
    for t in ("f32", "bf16", "f16"):
        eight = t != "f32" and m > 32
        e = ((2.0 ** -10 if eight else 0.0) + (k + 2) * 2.0 ** -23)
        tol = 1.13 * e * S[0] * (np.abs(U) + e * S[1]) + np.abs(G) * e * S[1] + np.abs(G * U) * (8 + np.minimum(4 * np.abs(G), 90)) * 2.0 ** -22 + HALF[t] * np.abs(H) + 2.0 ** -24
        got = pvq.pvq_fp8_gated(X, GATE, UP, act, DTYPES[t])
        assert (np.abs(f64(got) - H) <= tol).all(), (t, np.abs(f64(got) - H).max())
        out = matrix(np.zeros((m, n)), t, 3, 1)
        assert torch.equal(pvq.pvq_fp8_gated(X, GATE, UP, act, out=out), got)
        hats[t] = tol
    # kept products: codes of sums of 32 bits.  Half a step (2^-4, or 2^-10 of the scale) from the sum, whose own error can move
    # the scale of a block too: a step of twice the size
    e = (k + 2) * 2.0 ** -23
    for t in ("bf16", "f32"):
        h, gk, uk = pvq.pvq_fp8_gated(X, GATE, UP, act, DTYPES[t], keep=True)
        assert (np.abs(f64(h) - H) <= hats[t]).all()
        for b, want, s in ((gk, G, S[0]), (uk, U, S[1])):
            C, E = ref.planes(m, n)
            assert tuple(b.codes.shape) == (m, C) and tuple(b.exponents.shape) == (m, E)
            assert not b.codes[:, n:].any() and not b.exponents[:, C // 128:].any()
            wc, we = ref.encode(want)
            scale = np.ldexp(1.0, np.repeat(we[:, :C // 128].astype(int) - 127, 128, axis=1))[:, :n]
            value = f64(pvq.pvq_fp8_decode(b, torch.float32))
            assert (np.abs(value - want) <= np.maximum(2.0 ** -4 * np.abs(want), 2.0 ** -9 * scale) * 1.001 + e * s).all()
            # nearly all codes are those of the exact sums
            assert (b.codes.cpu().numpy() != wc).mean() <= 0.02 and (b.exponents.cpu().numpy() != we).mean() <= 0.1
    # H in blocks
    hb = pvq.pvq_fp8_gated(X, GATE, UP, act, encode=True)
    assert (hb.rows, hb.cols) == (m, n) and not hb.codes[:, n:].any()
    wc, we = ref.encode(H)
    scale = np.ldexp(1.0, np.repeat(we[:, :wc.shape[1] // 128].astype(int) - 127, 128, axis=1))[:, :n]
    e = 2.0 ** -10 + (k + 2) * 2.0 ** -23
    tol = 1.13 * e * S[0] * (np.abs(U) + e * S[1]) + np.abs(G) * e * S[1] + np.abs(G * U) * (8 + np.minimum(4 * np.abs(G), 90)) * 2.0 ** -22
    assert (np.abs(f64(pvq.pvq_fp8_decode(hb, torch.float32)) - H) <= np.maximum(2.0 ** -4 * np.abs(H), 2.0 ** -9 * scale) * 1.001 + tol * 1.1).all()


def test_activations_at_their_ends():
    # one input of one: G and U are the weights themselves
    g = np.array([0.0, -0.0, 1e-30, -1e-30, 1, -1, 5, -5, 16, -16, 20, -20, 88, -88, 200, -200, 1e4, -1e4, 1e30, -1e30])[:, None]
    X = pvq.pvq_fp8_encode(torch.ones(2, 1, device="cuda"))
    W, ONE = pvq.pvq_fp8_encode(dev(g.astype(np.float32))), pvq.pvq_fp8_encode(torch.ones(len(g), 1, device="cuda"))
    held = f64(pvq.pvq_fp8_decode(W, torch.float32))[:, 0]
    for act in ("silu", "gelu"):
        with np.errstate(over="ignore", invalid="ignore"):
            value, slope = ref.act(act, np.clip(held, -1e3, 1e3))
        value, slope = np.where(held < -1e3, 0, np.where(held > 1e3, held, value)), np.where(np.abs(held) > 1e3, held > 0, slope)
        h, gk, uk = pvq.pvq_fp8_gated(X, W, ONE, act, torch.float32, keep=True)
        assert np.allclose(f64(h)[0], value, rtol=1e-5, atol=1e-6)
        # dX = dG g + dU u with dH = 1, U = 1: slope and value, rounded to bfloat16 and multiplied out
        # (the twenty units of a token are one block, of scale 2^91, whose smallest code is 2^82: the others are kept as zeros)
        kept = f64(pvq.pvq_fp8_decode(gk, torch.float32))[0]
        assert np.array_equal(kept, ref.decode(*ref.encode(held[None]), len(g))[0])
        dh = torch.ones(2, len(g), dtype=torch.bfloat16, device="cuda")
        _, dgate, dup = pvq.pvq_fp8_gated_backward(dh, X, W, ONE, gk, uk, act, torch.float32)
        with np.errstate(over="ignore", invalid="ignore"):
            value, slope = ref.act(act, np.clip(kept, -1e3, 1e3))
        value, slope = np.where(kept < -1e3, 0, np.where(kept > 1e3, kept, value)), np.where(np.abs(kept) > 1e3, kept > 0, slope)
        assert np.allclose(f64(dgate)[:, 0], 2 * slope, rtol=2.0 ** -8 + 1e-5, atol=1e-5)
        assert np.allclose(f64(dup)[:, 0], 2 * value, rtol=2.0 ** -8 + 1e-5, atol=1e-5)


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_slopes_of_kept_values_at_their_ends(act):
    # one unit, a block for each token: dX = dH (U act'(G) Wg + act(G) Wu) with Wg = 1 and Wu = 0, then the other way round
    g = np.array([0.0, -0.0, 1e-30, -1e-30, 0.5, 1, -1, -1.25, 5, -5, 16, -16, 20, -20, 88, -88, 200, -200, 1e4, -1e4, 1e30, -1e30])[:, None]
    m = len(g)
    G, U = pvq.pvq_fp8_encode(dev(g.astype(np.float32))), pvq.pvq_fp8_encode(torch.ones(m, 1, device="cuda"))
    held = f64(pvq.pvq_fp8_decode(G, torch.float32))[:, 0]
    value, slope = ref.act(act, np.clip(held, -1e2, 1e2))
    value, slope = np.where(np.abs(held) > 1e2, np.maximum(held, 0), value), np.where(np.abs(held) > 1e2, held > 0, slope)
    X = pvq.pvq_fp8_encode(torch.ones(m, 1, device="cuda"))
    dh = torch.ones(m, 1, dtype=torch.bfloat16, device="cuda")
    one, zero = pvq.pvq_fp8_encode(torch.ones(1, 1, device="cuda")), pvq.pvq_fp8_encode(torch.zeros(1, 1, device="cuda"))
    for weights, want in (((one, zero), slope), ((zero, one), value)):
        dx, _, _ = pvq.pvq_fp8_gated_backward(dh, X, *weights, G, U, act, torch.float32, weight_grads=False)
        # rounded to bfloat16 once; the float32 arithmetic in front is a few places of terms of the size of 1 + |g sigma|
        assert np.allclose(f64(dx)[:, 0], want, rtol=2.0 ** -8 + 1e-5, atol=1e-5)


BACKWARD = [(1, 1, 1), (2, 130, 128), (33, 100, 129), (70, 129, 385), (130, 300, 200), (300, 64, 513)]


@pytest.mark.parametrize("m,n,k", BACKWARD)
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_gated_backward(m, n, k, act, dtype):
    rng = np.random.default_rng(m + 100 * n + 10000 * k)
    xc, xe, x = ref.random_blocks(rng, m, k)
    gc, ge, g = ref.random_blocks(rng, n, k, k ** -0.5)
    uc, ue, u = ref.random_blocks(rng, n, k, k ** -0.5)
    Gc, Ge, G = ref.random_blocks(rng, m, n)
    Uc, Ue, U = ref.random_blocks(rng, m, n)
    dh_t = matrix(rng.standard_normal((m, n)), "bf16", 3 if n % 2 else 8, 1 if n % 2 else 0)
    dh = f64(dh_t)
    value, slope = ref.act(act, G)
    dU, dG = dh * value, dh * U * slope
    # dG and dU: half a step of bfloat16, and the float32 arithmetic and the activation in front of it
    tU = np.abs(dh * G) * (12 + np.minimum(4 * np.abs(G), 90)) * 2.0 ** -22 + 2.0 ** -8 * np.abs(dU)
    tG = np.abs(dh * U) * (1 + np.abs(G)) * (16 + np.minimum(4 * np.abs(G), 90)) * 2.0 ** -22 + 2.0 ** -8 * np.abs(dG)
    args = (dh_t, blocks(xc, xe, k), blocks(gc, ge, k), blocks(uc, ue, k), blocks(Gc, Ge, n), blocks(Uc, Ue, n), act, DTYPES[dtype])
    got = pvq.pvq_fp8_gated_backward(*args)
    a = np.abs
    wants = ((dG @ g + dU @ u, tG @ a(g) + tU @ a(u), a(dG) @ a(g) + a(dU) @ a(u), 2 * n), (dG.T @ x, tG.T @ a(x), a(dG).T @ a(x), m),
             (dU.T @ x, tU.T @ a(x), a(dU).T @ a(x), m))
    for v, (want, off, size, K) in zip(got, wants):
        tol = 1.01 * off + (K + 2) * 2.0 ** -23 * 1.01 * size + HALF[dtype] * (a(want) + off) + 2.0 ** -24
        assert (a(f64(v) - want) <= tol).all()
        # roundings of dG and dU to bfloat16 are random: 2^-8 of the root of the squares, not of the sum
        assert np.linalg.norm(f64(v) - want) <= (2.0 ** -8 + HALF[dtype] + 1e-4) * max(np.linalg.norm(want), np.linalg.norm(size) / np.sqrt(K)) + 2.0 ** -24 * np.sqrt(want.size)
    only_x = pvq.pvq_fp8_gated_backward(*args, weight_grads=False)
    only_w = pvq.pvq_fp8_gated_backward(*args, input_grad=False)
    assert torch.equal(only_x[0], got[0]) and only_x[1] is None and only_x[2] is None
    assert only_w[0] is None and torch.equal(only_w[1], got[1]) and torch.equal(only_w[2], got[2])


def test_gradients_are_the_differences_of_the_forward_pass():
    """d(sum H) along a direction of the inputs and of the weights, by central differences of the 64-bit forward pass around the
    stored values; kept products in 8 bits are 2^-4 off each at most, which is random over the sum."""
    rng = np.random.default_rng(3)
    m, n, k = 40, 150, 200
    xc, xe, x = ref.random_blocks(rng, m, k)
    gc, ge, g = ref.random_blocks(rng, n, k, k ** -0.5)
    uc, ue, u = ref.random_blocks(rng, n, k, k ** -0.5)
    weight = f64(torch.from_numpy(rng.standard_normal((m, n))).bfloat16())
    for act in ("silu", "gelu"):
        X, GATE, UP = blocks(xc, xe, k), blocks(gc, ge, k), blocks(uc, ue, k)
        _, G, U = pvq.pvq_fp8_gated(X, GATE, UP, act, torch.bfloat16, keep=True)
        dx, dg, du = (f64(t) for t in pvq.pvq_fp8_gated_backward(dev(weight).bfloat16(), X, GATE, UP, G, U, act, torch.float32))
        for value, grad, which in ((x, dx, 0), (g, dg, 1), (u, du, 2)):
            d, h = rng.standard_normal(value.shape), 1e-5
            side = []
            for s in (h, -h):
                parts = [x, g, u]
                parts[which] = value + s * d
                side.append((weight * gated_reference(*parts, act)[2]).sum())
            difference = (side[0] - side[1]) / (2 * h)
            assert abs((grad * d).sum() - difference) <= 0.05 * np.linalg.norm(grad) + 1e-6


def test_a_feed_forward_block_from_packed_weights():
    """Packed weights decoded to bfloat16, put into 8-bit blocks, and multiplied with a prompt, forward and backward, against the same
    chain in 64 bits; the few first tokens against the product on the packed weights."""
    hidden, inner, tokens = 256, 384, 70
    D, K = 8, pvq.pvq_max_k(8, 24)
    ctx = pvq.pvq_ctx_create(D, K)
    rng = np.random.default_rng(11)
    dense, packed, W = [], [], []
    for i, (rows, cols) in enumerate(((inner, hidden), (inner, hidden), (hidden, inner))):
        wf, wb = si.gaussian_weights(rows, cols, 0.06, seed=si.BASE_SEED + 950 + i, bf16=True)
        packed.append(pvq.pvq_encode(ctx, gu.to_dev_bf16(wb)))
        dense.append(pvq.pvq_decode(ctx, packed[-1], torch.bfloat16))
        W.append(pvq.pvq_fp8_encode(dense[-1]))
    x_t = dev(rng.standard_normal((tokens, hidden))).bfloat16()
    signs = torch.zeros(hidden, dtype=torch.uint8, device="cuda")
    X = pvq.pvq_fp8_encode(pvq.pvq_hadamard(pvq.pvq_hadamard(x_t, 256, signs), 256, signs, inverse=True))
    x, w = f64(pvq.pvq_fp8_decode(X, torch.float32)), [f64(pvq.pvq_fp8_decode(b, torch.float32)) for b in W]
    h, G, U = pvq.pvq_fp8_gated(X, W[0], W[1], "silu", torch.bfloat16, keep=True)
    H = pvq.pvq_fp8_encode(h)
    y = pvq.pvq_fp8_product(H, W[2], torch.bfloat16)
    _, _, h64 = gated_reference(x, w[0], w[1], "silu")
    hq = f64(pvq.pvq_fp8_decode(H, torch.float32))
    assert np.linalg.norm(hq - h64) <= 2.0 ** -4 * np.linalg.norm(h64)              # half a step of e4m3
    y64 = hq @ w[2].T
    assert np.linalg.norm(f64(y) - y64) <= (2.0 ** -8 + 4e-4) * np.linalg.norm(y64)
    # serving: H straight into blocks, and one token at a time
    hb = pvq.pvq_fp8_gated(X, W[0], W[1], "silu", encode=True)
    assert np.linalg.norm(f64(pvq.pvq_fp8_decode(hb, torch.float32)) - h64) <= 2.0 ** -4 * np.linalg.norm(h64)
    one = pvq.Fp8Blocks(1, hidden, X.codes[5:6], X.exponents[5:6])
    h1 = pvq.pvq_fp8_gated(one, W[0], W[1], "silu", torch.bfloat16)
    assert np.linalg.norm(f64(h1)[0] - h64[5]) <= (2.0 ** -8 + 1e-4) * np.linalg.norm(h64[5])
    # 16 tokens on the packed weights: both sides' weights and activations are rounded to e4m3 here, half a step 2^-4 each at most
    gemv = f64(pvq.pvq_decode_gemv(ctx, packed[0], x_t[:16].contiguous()))
    wide = f64(pvq.pvq_fp8_product(pvq.Fp8Blocks(16, hidden, X.codes[:16], X.exponents[:16]), W[0], torch.float32))
    assert np.linalg.norm(wide - gemv) <= (2 * 2.0 ** -4 + 2.0 ** -8) * np.linalg.norm(gemv)
    # backward through both halves
    dy = dev(rng.standard_normal((tokens, hidden))).bfloat16()
    dh = pvq.pvq_fp8_input_grad(dy, W[2], torch.bfloat16)
    dw2 = pvq.pvq_fp8_weight_grad(dy, H, torch.float32)
    assert np.linalg.norm(f64(dh) - f64(dy) @ w[2]) <= (2.0 ** -8 + 1e-4) * np.linalg.norm(f64(dy) @ w[2])
    assert np.linalg.norm(f64(dw2) - f64(dy).T @ hq) <= 1e-5 * np.linalg.norm(f64(dy).T @ hq)
    dx, dgate, dup = pvq.pvq_fp8_gated_backward(dh, X, W[0], W[1], G, U, "silu", torch.bfloat16)
    g64, u64 = f64(pvq.pvq_fp8_decode(G, torch.float32)), f64(pvq.pvq_fp8_decode(U, torch.float32))
    value, slope = ref.act("silu", g64)
    dU, dG = f64(dh) * value, f64(dh) * u64 * slope
    for got, want in ((dx, dG @ w[0] + dU @ w[1]), (dgate, dG.T @ x), (dup, dU.T @ x)):
        assert np.linalg.norm(f64(got) - want) <= 2 * 2.0 ** -8 * np.linalg.norm(want)
    ctx.close()


def everything(X, GATE, UP, dh, x_t):
    """All entries once, on the current stream."""
    b = pvq.pvq_fp8_encode(x_t)
    h, G, U = pvq.pvq_fp8_gated(X, GATE, UP, "silu", torch.bfloat16, keep=True)
    hb = pvq.pvq_fp8_gated(X, GATE, UP, "gelu", encode=True)
    few = pvq.Fp8Blocks(5, X.cols, X.codes[:5], X.exponents[:5])
    return [b.codes, b.exponents, pvq.pvq_fp8_decode(b, torch.float16), h, G.codes, U.codes, hb.codes, pvq.pvq_fp8_product(X, GATE, torch.bfloat16),
            pvq.pvq_fp8_product(X, GATE, torch.float32), pvq.pvq_fp8_product(few, GATE), pvq.pvq_fp8_gated(few, GATE, UP), pvq.pvq_fp8_input_grad(dh, GATE, torch.bfloat16),
            pvq.pvq_fp8_weight_grad(dh, X, torch.float32), *pvq.pvq_fp8_gated_backward(dh, X, GATE, UP, G, U, "silu", torch.bfloat16)]


def inputs(seed, m=200, n=300, k=520):
    rng = np.random.default_rng(seed)
    X, GATE, UP = (blocks(*ref.random_blocks(rng, r, k, s)[:2], k) for r, s in ((m, 1.0), (n, k ** -0.5), (n, k ** -0.5)))
    return X, GATE, UP, dev(rng.standard_normal((m, n))).bfloat16(), dev(rng.standard_normal((m, k))).bfloat16()


def test_in_a_graph_and_on_two_streams():
    first, second = inputs(1), inputs(2)
    want = [[t.clone() for t in everything(*i)] for i in (first, second)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [None, None]
    for _ in range(3):
        for i, s in enumerate(streams):
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                got[i] = everything(*(first, second)[i])
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert all(torch.equal(x, y) for x, y in zip(a, b))
    # two graphs, replayed several times with eager work between, their inputs changed in place
    graphs = []
    for i in (first, second):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = everything(*i)
        graphs.append((g, out))
    for turn in range(4):
        for (g, out), w, i in zip(graphs, want, (first, second)):
            for t in out:
                t.fill_(1)
            g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(x, y) for x, y in zip(out, w)), turn
        eager = everything(*first)
        assert all(torch.equal(x, y) for x, y in zip(eager, want[0]))
    X = first[0]
    X.codes.copy_(second[0].codes)
    X.exponents.copy_(second[0].exponents)
    changed = [t.clone() for t in everything(*first)]
    graphs[0][0].replay()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(graphs[0][1], changed))


def test_the_binding_checks_shapes():
    X, GATE, UP, dh, x_t = inputs(4)
    short = pvq.Fp8Blocks(X.rows, X.cols, X.codes[:, :512].contiguous(), X.exponents)
    for call in (lambda: pvq.pvq_fp8_decode(short), lambda: pvq.pvq_fp8_product(short, GATE), lambda: pvq.pvq_fp8_weight_grad(dh[:-1], X),
                 lambda: pvq.pvq_fp8_decode(pvq.Fp8Blocks(X.rows, X.cols, X.codes.to(torch.int16), X.exponents)),
                 lambda: pvq.pvq_fp8_input_grad(dh[:, :-1], GATE), lambda: pvq.pvq_fp8_input_grad(dh.float(), GATE),
                 lambda: pvq.pvq_fp8_product(X, GATE, out=torch.empty(2, 2, device="cuda")), lambda: pvq.pvq_fp8_encode(x_t.t()),
                 lambda: pvq.pvq_fp8_product(X, GATE, out=torch.empty(300, 200, device="cuda").t()),
                 lambda: pvq.pvq_fp8_encode(x_t[:1].expand(4, -1)),
                 lambda: pvq.pvq_fp8_product(X, pvq.Fp8Blocks(GATE.rows, GATE.cols, GATE.codes.cpu(), GATE.exponents)),
                 lambda: pvq.pvq_fp8_gated_backward(dh, X, GATE, UP, X, X)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(KeyError):
        pvq.pvq_fp8_encode(x_t.double())
    with pytest.raises(KeyError):
        pvq.pvq_fp8_product(X, GATE, torch.float64)


def test_offsets_beyond_32_bits():
    """Planes and results of more than 4 GiB: the last rows are those of a small call."""
    m, n, k = 40, 70, 384
    rng = np.random.default_rng(8)
    (xc, xe, x), (wc, we, w) = ref.random_blocks(rng, m, k), ref.random_blocks(rng, n, k)
    X, W = blocks(xc, xe, k), blocks(wc, we, k)
    rows = (1 << 32) // k + 1000
    codes, exps = torch.zeros(rows, k, dtype=torch.uint8, device="cuda"), torch.full((rows, 4), 127, dtype=torch.uint8, device="cuda")
    codes[-n:], exps[-n:] = W.codes, W.exponents
    LONG = pvq.Fp8Blocks(rows, k, codes, exps)
    # (which instruction forms the sums depends on the shape: both are as far from the 64-bit ones as the 8-bit one may be)
    got, want = pvq.pvq_fp8_product(X, LONG, torch.bfloat16), pvq.pvq_fp8_product(X, W, torch.bfloat16)
    for v in (got[:, -n:], want):
        check_sum(v, x @ w.T, np.abs(x) @ np.abs(w).T, k, "bf16", True, np.sqrt((x * x) @ (w * w).T))
    assert not got[:, :1000].any()
    X = pvq.Fp8Blocks(7, k, X.codes[:7], X.exponents[:7])
    assert torch.equal(pvq.pvq_fp8_product(X, LONG, torch.bfloat16)[:, -n:], pvq.pvq_fp8_product(X, W, torch.bfloat16))      # few rows
    del got
    got = pvq.pvq_fp8_product(LONG, W, torch.bfloat16)                  # tiles, and a result of 1.5 GiB
    want = pvq.pvq_fp8_product(pvq.Fp8Blocks(n, k, W.codes, W.exponents), W, torch.float32)
    assert torch.allclose(got[-n:].float(), want, rtol=2.0 ** -7, atol=0.05) and not got[:1000].any()
    del got
    values = pvq.pvq_fp8_decode(LONG, torch.bfloat16)                    # 8 GiB
    assert torch.equal(values[-n:], pvq.pvq_fp8_decode(W, torch.bfloat16))
    back = pvq.pvq_fp8_encode(values)
    assert torch.equal(pvq.pvq_fp8_decode(pvq.Fp8Blocks(n, k, back.codes[-n:], back.exponents[-n:]), torch.bfloat16), values[-n:])
    del back, values
    dy = torch.zeros(rows, 40, dtype=torch.bfloat16, device="cuda")
    dy[-n:] = torch.from_numpy(rng.standard_normal((n, 40)))
    dw = pvq.pvq_fp8_weight_grad(dy, LONG, torch.float32)                 # over all rows, of which the last count
    few = pvq.pvq_fp8_weight_grad(dy[-n:], W, torch.float32)
    assert torch.allclose(dw, few, rtol=1e-4, atol=1e-4)
