"""How exact the sums behind results of 8-bit blocks are, closely enough to tell the two matrix instructions apart.

A sum of K random terms, r the root of their squares' sum:
  - bfloat16 instruction: float32 sums, off by at most sqrt(K) 2^-23 r in the mean square (tests/test_gpu_fp8.py).
  - 8-bit instruction: of eight products those bits are dropped that lie 14 binary places below the largest one's exponent, a term's error is uniform over
    an interval of 2^-14 times the largest, which of eight Gaussian products is below three standard deviations on average: 3 * 2^-14 / sqrt(12) < 2^-14
    of a term's standard deviation, so 2^-14 r in all (3.3e-5 measured, 0.55 of that), beside the float32 sum's own error.
Results are rounded.  A sum that is off by e is rounded otherwise than the exact one if a border between two values lies between them: with
probability |e| / (distance of borders).  So the share of results that differ from the rounded exact sums is at most the mean of
e / step, and it tells an e ten times as large even where that is hidden in the roundings' own size."""
import numpy as np
import pytest

import paper_2410_16926_amd as pvq
from tests import fp8_reference as ref
from tests import test_gpu_fp8 as base

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
EIGHT_BIT = 2.0 ** -14


def float32_sums(k):
    return np.sqrt(k) * 2.0 ** -23


def gaussian(seed, *shapes):
    """Gaussian matrices in blocks, and what they hold in float64 on the GPU."""
    rng = np.random.default_rng(seed)
    out = []
    for rows, cols, scale in shapes:
        c, e = ref.encode(rng.standard_normal((rows, cols)) * scale)
        out.append((base.blocks(c, e, cols), torch.from_numpy(ref.decode(c, e, cols)).cuda()))
    return out


def times(a, b):
    """a b^T in 64 bits, and the root of the sums of the squared terms."""
    return torch.matmul(a, b.T.contiguous()), torch.matmul(a * a, (b * b).T.contiguous()).sqrt()


def steps16(y):
    """The distance of neighbouring float16 values at y."""
    return torch.ldexp(torch.ones_like(y), (torch.frexp(y)[1] - 11).clamp(min=-24))


def differing(got, y, off):
    """(share of float16 results that are not the rounded y, at most how many may be where y is `off` off)"""
    return (got != y.half()).double().mean().item(), (off / steps16(y)).clamp(max=1).mean().item()


# (shape, kind of tile, whether it is split)
@pytest.mark.parametrize("m,n,k,kind,split", [(1316, 4457, 66, "tiles_8bit", False), (1024, 3000, 2048, "tiles_8bit", False), (72, 4359, 4739, "tiles_8bit", True),
                                              (200, 300, 520, "tiles_64", False), (64, 1500, 1500, "tiles_64", True), (20, 3000, 1500, "rows", False)])
def test_a_products_sums(m, n, k, kind, split):
    plan = pvq.pvq_fp8_plan("product", m, n, k, 1)
    assert plan[0] == kind and (plan[1] > 1) == split
    (A, a), (B, b) = gaussian(k, (m, k, 1.0), (n, k, 1.0))
    y, root = times(a, b)
    off = float32_sums(k) + (EIGHT_BIT if kind == "tiles_8bit" else 0.0)
    share, most = differing(pvq.pvq_fp8_product(A, B, torch.float16), y, off * root)
    assert share <= most, (share, most)
    # float32 results have none but the float32 sum's error, whatever the shape
    d = pvq.pvq_fp8_product(A, B, torch.float32).double() - y
    assert d.norm() <= float32_sums(k) * root.norm() + 2.0 ** -24 * y.norm()


@pytest.mark.parametrize("m,n,k", [(72, 4359, 4739), (4273, 265, 4714)])
def test_a_split_products_sums_before_they_are_rounded(m, n, k):
    """The parts' float32 sums as they lie in the workspace, added in 64 bits."""
    kind, parts = pvq.pvq_fp8_plan("product", m, n, k)
    assert kind == "tiles_8bit" and parts > 1
    (A, a), (B, b) = gaussian(k, (m, k, 1.0), (n, k, 1.0))
    y, root = times(a, b)
    out = torch.empty(m, n, dtype=torch.bfloat16, device="cuda")
    work = torch.zeros(parts, m, n, device="cuda")
    status = pvq.lib().pvq_fp8_product(A.codes.data_ptr(), A.exponents.data_ptr(), m, B.codes.data_ptr(), B.exponents.data_ptr(), n, k, out.data_ptr(), 2, n,
                                       work.data_ptr(), work.numel() * 4, torch.cuda.current_stream().cuda_stream)
    assert status == 0
    assert torch.equal(out, pvq.pvq_fp8_product(A, B, torch.bfloat16))
    d = work.double().sum(0) - y
    assert d.norm() <= (EIGHT_BIT + float32_sums(k)) * root.norm()


@pytest.mark.parametrize("m,n,k,kind", [(1316, 4457, 66, "tiles_8bit"), (132, 5637, 4311, "tiles_8bit"), (64, 1500, 1500, "tiles_64"), (20, 1500, 1500, "rows")])
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_a_gated_blocks_sums(m, n, k, kind, act):
    """An error e of G and U becomes act'(G) U e + act(G) e, and the activation's arithmetic is (8 + 4 |G|) 2^-22 of H as in tests/test_gpu_fp8.py."""
    assert pvq.pvq_fp8_plan("gated", m, n, k, 1)[0] == kind
    (X, x), (W, w), (V, v) = gaussian(k, (m, k, 1.0), (n, k, k ** -0.5), (n, k, k ** -0.5))
    (G, rg), (U, ru) = times(x, w), times(x, v)
    value, slope = (torch.from_numpy(t).cuda() for t in ref.act(act, G.cpu().numpy()))
    e = float32_sums(k) + (EIGHT_BIT if kind == "tiles_8bit" else 0.0)
    off = e * ((slope * U).abs() * rg + value.abs() * ru) + (8 + 4 * G.abs()) * 2.0 ** -22 * (value * U).abs()
    share, most = differing(pvq.pvq_fp8_gated(X, W, V, act, torch.float16), value * U, off)
    assert share <= most, (share, most)


@pytest.mark.parametrize("m,n,k,kind", [(1316, 4457, 66, "tiles_256"), (2306, 1250, 65, "tiles_256"), (132, 5637, 4311, "tiles_256"), (64, 1500, 1500, "tiles_64"),
                                        (20, 1500, 1500, "tiles_64")])
@pytest.mark.parametrize("dtype", ["bf16", "f32", "f16"])
def test_kept_products_are_codes_of_float32_sums(m, n, k, kind, dtype):
    """Whatever H is.  (The 8-bit instruction would change one code of 2000.)  Codes lie 2^-3 of a value's power of two apart, below 2^-6 of the scale 2^-9
    of it; a block's scale changes where its largest value is that close to 448 times a power of two.

    A sum of K terms in P parts: the partial sum of i terms of a part is r sqrt(i / K) in the mean square, and each addition is off by at most 2^-23 of it,
    at random; the sum over i up to K / P of 2^-46 r^2 i / K is 2^-46 r^2 K / (2 P^2), and that of all parts 2^-46 r^2 K / (2 P): 2^-23 sqrt(K / (2 P)) r."""
    plan, parts = pvq.pvq_fp8_plan("gated_kept", m, n, k, {"f32": 0, "f16": 1, "bf16": 2}[dtype])
    assert plan == kind
    (X, x), (W, w), (V, v) = gaussian(k, (m, k, 1.0), (n, k, k ** -0.5), (n, k, k ** -0.5))
    _, G, U = pvq.pvq_fp8_gated(X, W, V, "silu", base.DTYPES[dtype], keep=True)
    for kept, weights in ((G, w), (U, v)):
        y, root = (t.cpu().numpy() for t in times(x, weights))
        codes, exps = ref.encode(y)
        got_codes, got_exps = kept.codes.cpu().numpy(), kept.exponents.cpu().numpy()
        per = codes.shape[1] // 128
        agree = got_exps[:, :per] == exps[:, :per]
        assert (~agree).mean() <= 1e-4
        scale = np.ldexp(1.0, np.repeat(exps[:, :per].astype(int) - 127, 128, axis=1))[:, :n]
        step = np.maximum(np.ldexp(1.0, np.frexp(y)[1] - 4), 2.0 ** -9 * scale)
        most = np.minimum(2.0 ** -23 * np.sqrt(k / (2 * parts)) * root / step, 1).mean()
        share = ((got_codes != codes) & np.repeat(agree, 128, axis=1))[:, :n].mean()
        assert most < 2.5e-4                     # (or it would not tell the 8-bit instruction)
        assert share <= most, (share, most)
