"""How far results of 8-bit blocks may be off where a format in between could hold fewer bits than the result.  Reference in 64 bits
(tests/fp8_reference.py); h(t) = eps / 2 of a type is half a step relative to a value."""
import numpy as np
import pytest

import paper_2410_16926_amd as pvq
from tests import fp8_reference as ref
from tests import test_gpu_fp8 as base

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def backward_inputs(m, n, k, seed=0):
    """(arguments of the backward pass but the activation and the type, their values in 64 bits)"""
    rng = np.random.default_rng(m + 100 * n + 10000 * k + seed)
    planes = [ref.random_blocks(rng, *a) for a in ((m, k), (n, k, k ** -0.5), (n, k, k ** -0.5), (m, n), (m, n))]
    dh = base.matrix(rng.standard_normal((m, n)), "bf16", 3 if n % 2 else 8, 1 if n % 2 else 0)
    return (dh, *(base.blocks(c, e, v.shape[1]) for c, e, v in planes)), (base.f64(dh), *(v for _, _, v in planes))


# each length of a sum of one step of 64, of whole ones and of a few values more, in small and in large tiles
@pytest.mark.parametrize("m,n,k", [(1, 1, 1), (2, 130, 128), (33, 100, 129), (64, 128, 256), (70, 129, 385), (300, 64, 513), (130, 2000, 70), (2000, 130, 70), (517, 1409, 1024),
                                   (65, 4609, 1625), (2857, 4108, 67), (5513, 72, 1291), (75, 2309, 3120), (1000, 2100, 1200)])
@pytest.mark.parametrize("act,dtype", [("silu", "f32"), ("gelu", "f32"), ("silu", "f16")])
def test_gradients_of_the_gated_block_have_the_bits_of_their_type(m, n, k, act, dtype):
    """dG and dU in two pieces of bfloat16: v = hi + lo + r, |v - hi| <= 2^-8 |v| and exact in float32, so |r| <= 2^-8 |v - hi| <= 2^-16 |v|.
    The float32 arithmetic of act in front of it is a few places, more of them for large arguments; sums of K terms as in
    tests/test_gpu_fp8.py, a term for each piece.  In the 2-norm the roundings are random over the sum; the arithmetic's
    bound for arguments of the size of the data (|G| up to 8: 12 + 32 places of 2^-22) is 2^-16 once more."""
    args, (dh, x, g, u, G, U) = backward_inputs(m, n, k)
    value, slope = ref.act(act, G)
    dU, dG = dh * value, dh * U * slope
    a = np.abs
    tU = a(dh * G) * (12 + np.minimum(4 * a(G), 90)) * 2.0 ** -22 + 2.0 ** -16 * a(dU)
    tG = a(dh * U) * (1 + a(G)) * (16 + np.minimum(4 * a(G), 90)) * 2.0 ** -22 + 2.0 ** -16 * a(dG)
    half = base.HALF[dtype]
    wants = ((dG @ g + dU @ u, tG @ a(g) + tU @ a(u), a(dG) @ a(g) + a(dU) @ a(u), np.sqrt((dG * dG) @ (g * g) + (dU * dU) @ (u * u)), 4 * n),
             (dG.T @ x, tG.T @ a(x), a(dG).T @ a(x), np.sqrt((dG * dG).T @ (x * x)), 2 * m), (dU.T @ x, tU.T @ a(x), a(dU).T @ a(x), np.sqrt((dU * dU).T @ (x * x)), 2 * m))
    got = pvq.pvq_fp8_gated_backward(*args, act, base.DTYPES[dtype])
    for v, (want, off, size, root, K) in zip(got, wants):
        d = base.f64(v) - want
        assert (a(d) <= 1.01 * off + (K + 2) * 2.0 ** -23 * 1.01 * size + half * (a(want) + off) + 2.0 ** -24).all()
        assert np.linalg.norm(d) <= (2 * 2.0 ** -16 + np.sqrt(K) * 2.0 ** -23 + half) * np.linalg.norm(root) + 2.0 ** -24 * np.sqrt(want.size)
    assert all(torch.equal(p, q) for p, q in zip(got, pvq.pvq_fp8_gated_backward(*args, act, base.DTYPES[dtype])))


@pytest.mark.parametrize("dh,dgate,dup", [(np.inf, np.inf, np.inf), (-np.inf, -np.inf, -np.inf), (np.nan, np.nan, np.nan), (2.0 ** 126, 2.0 ** 126, np.inf),
                                          (186 / 128 * 2.0 ** 121, 186 / 128 * 2.0 ** 121, np.inf), (2.0 ** -120, 2.0 ** -120, 88 * 2.0 ** -120)])
def test_slopes_at_the_ends_of_the_type(dh, dgate, dup):
    """One unit of one token, with G = 88 (act(G) = G, act' = 1) and U = 1.  The second piece of an infinity is nothing, not infinity - infinity;
    so is that of 186 / 128 * 2^121 * 88 = 2046 / 1024 * 2^127, a float32 number that rounds out of bfloat16."""
    def one(v):
        return pvq.pvq_fp8_encode(torch.full((1, 1), v, device="cuda"))
    dh = torch.full((1, 1), dh, device="cuda").bfloat16()
    for act in ("silu", "gelu"):
        _, got_gate, got_up = pvq.pvq_fp8_gated_backward(dh, one(1.0), one(1.0), one(1.0), one(88.0), one(1.0), act, torch.float32)
        assert np.array_equal([float(got_gate), float(got_up)], [dgate, dup], equal_nan=True)
