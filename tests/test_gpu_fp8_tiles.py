"""8-bit blocks at the sizes that decide how the products' kernels divide their work: sums that are split into parts, more tiles than
compute units (a workgroup goes from one to the next), low tiles and whole ones, few rows and one more.  The checks and their
tolerances are those of tests/test_gpu_fp8.py."""
import numpy as np
import pytest

import paper_2410_16926_amd as pvq
from tests import fp8_reference as ref
from tests import test_gpu_fp8 as base

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

# (also small tiles against large ones: up to some 10^10 operations, or where large ones would be few)
# few tiles of a long sum; either side of 8, 16 and 32 rows; a tile and one row more; 274 tiles of few rows and 289 of many
PRODUCTS = [(33, 100, 20011), (70, 300, 20011), (300, 260, 6000), (8, 40, 1300), (9, 40, 1300), (16, 33, 20011), (32, 513, 1025), (33, 513, 1025),
            (128, 256, 513), (129, 257, 512), (256, 256, 640), (257, 255, 641), (100, 70001, 130), (4352, 4100, 130), (333, 3001, 11008), (1024, 3000, 2048), (700, 2050, 3001)]


# every kind of large tile: in one round or several, its sums whole or split
PRODUCTS += [(1316, 4457, 66), (4892, 3288, 64), (72, 4359, 4739), (3550, 842, 65), (66, 4305, 4576), (3667, 2164, 64), (5063, 3203, 66), (4273, 265, 4714)]


@pytest.mark.parametrize("m,n,k", PRODUCTS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_products(m, n, k, dtype):
    base.test_product(m, n, k, dtype)


@pytest.mark.parametrize("m,n,k,act", [(70, 200, 9000, "silu"), (40, 129, 5000, "gelu"), (32, 260, 4100, "silu"), (300, 17000, 129, "gelu"), (300, 3000, 4000, "silu"),
                                         (1100, 2100, 640, "gelu"), (20, 4000, 300, "gelu"),
                                         (82, 2052, 4799, "silu"), (68, 4737, 4996, "gelu"), (72, 4156, 2998, "gelu"), (132, 5637, 4311, "silu"),
                                         (1364, 5712, 64, "silu"), (2306, 1250, 65, "gelu"), (2578, 937, 64, "silu")])
def test_gated(m, n, k, act):
    base.test_gated(m, n, k, act)


# dX and dW of each: either's sum long and its tiles few; many tiles of few rows, and of many
@pytest.mark.parametrize("m,n,k,dtype,gap,shift", [(70, 20011, 300, "f32", 0, 0), (70, 20011, 300, "bf16", 5, 1), (20011, 70, 300, "f16", 0, 0),
                                                   (20011, 72, 300, "f32", 8, 0), (100, 130, 70001, "bf16", 0, 0), (4352, 64, 4100, "f32", 0, 0),
                                                   (65, 4352, 4100, "bf16", 3, 1), (128, 128, 256, "f16", 0, 0), (129, 192, 257, "f32", 0, 0),
                                                   (333, 3001, 2100, "bf16", 0, 0), (700, 1100, 3000, "f32", 5, 1), (517, 2000, 2048, "bf16", 8, 0), (64, 63, 65, "f32", 1, 0),
                                                   (63, 65, 64, "bf16", 0, 1), (1500, 1500, 1500, "f16", 4, 0),
                                                   (65, 661, 4588, "f32", 0, 0), (65, 2834, 5480, "bf16", 3, 1), (4658, 72, 4110, "f16", 0, 0), (5626, 66, 522, "f32", 0, 0),
                                                   (2898, 74, 5597, "bf16", 0, 0), (69, 4967, 4331, "f32", 1, 0), (5513, 72, 1291, "f16", 8, 0), (3132, 65, 5179, "f32", 0, 0),
                                                   (4208, 5227, 260, "bf16", 0, 0), (69, 4697, 3398, "f32", 8, 0), (5502, 4242, 258, "f32", 0, 1)])
def test_gradients_of_a_product(m, n, k, dtype, gap, shift):
    base.test_gradients_of_a_product(m, n, k, dtype, gap, shift)


@pytest.mark.parametrize("m,n,k,act,dtype", [(70, 9000, 129, "silu", "f32"), (9000, 70, 129, "gelu", "bf16"), (100, 130, 35001, "silu", "bf16"),
                                             (4352, 64, 4100, "gelu", "f32"), (65, 2304, 4100, "silu", "f16"), (500, 700, 3000, "gelu", "f32"), (1000, 2100, 1200, "silu", "bf16"), (64, 65, 4000, "silu", "f32"),
                                             (64, 5138, 270, "gelu", "bf16"), (75, 2309, 3120, "silu", "f32"), (4774, 65, 2185, "gelu", "f16"), (66, 4279, 801, "silu", "f32"),
                                             (65, 4609, 1625, "gelu", "bf16"), (2857, 4108, 67, "silu", "bf16"), (5626, 66, 522, "gelu", "f32"), (2898, 74, 5597, "silu", "bf16"),
                                             (74, 2414, 4227, "gelu", "f32"), (5513, 72, 1291, "silu", "f16"), (3132, 65, 5179, "silu", "f32"), (5471, 3078, 65, "gelu", "f32")])
def test_gated_backward(m, n, k, act, dtype):
    base.test_gated_backward(m, n, k, act, dtype)


@pytest.mark.parametrize("m,n", [(3, 5), (3001, 4001)])
def test_empty_sums_fill_the_result(m, n):
    none = [pvq.pvq_fp8_encode(torch.zeros(r, 0, device="cuda")) for r in (m, n)]
    for t in ("f32", "bf16"):
        out = base.matrix(np.ones((m, n)), t, 3, 1)
        assert not pvq.pvq_fp8_product(*none, out=out).any()
        assert torch.isnan(torch.as_strided(out, (m - 1, 3), (n + 3, 1), 1 + n)).all()


@pytest.mark.parametrize("m", [5, 70])
def test_nothing_is_taken_from_behind_the_last_exponent(m):
    """Three blocks of a row have four bytes of exponents: the fourth counts for nothing."""
    n, k = 150, 300
    rng = np.random.default_rng(m)
    planes = [ref.random_blocks(rng, r, k)[:2] for r in (m, n, n)]
    dy = base.dev(rng.standard_normal((m, n))).bfloat16()

    def all_of(last):
        b = []
        for c, e in planes:
            e = e.copy()
            e[:, 3] = last
            b.append(base.blocks(c, e, k))
        X, W, V = b
        h, G, U = pvq.pvq_fp8_gated(X, W, V, out_dtype=torch.bfloat16, keep=True)
        return [pvq.pvq_fp8_product(X, W, torch.bfloat16), pvq.pvq_fp8_product(X, W, torch.float32), pvq.pvq_fp8_gated(X, W, V), h, G.codes, U.codes,
                pvq.pvq_fp8_input_grad(dy, W), pvq.pvq_fp8_weight_grad(dy, X), pvq.pvq_fp8_decode(X), *pvq.pvq_fp8_gated_backward(dy, X, W, V, G, U)]
    want = all_of(0)
    for last in (127, 254, 255):
        assert all(torch.equal(x, y) for x, y in zip(all_of(last), want))


def test_split_sums_in_graphs_and_on_two_streams():
    """Two graphs whose splits' sums lie in workspaces of their own, replayed in turn and at once."""
    def inputs(seed, m=70, n=300, k=9000):
        rng = np.random.default_rng(seed)
        X, GATE, UP = (base.blocks(*ref.random_blocks(rng, r, k, s)[:2], k) for r, s in ((m, 1.0), (n, k ** -0.5), (n, k ** -0.5)))
        down = base.blocks(*ref.random_blocks(rng, k, n)[:2], n)
        return X, GATE, UP, down, base.dev(rng.standard_normal((m, k))).bfloat16()

    def run(X, GATE, UP, down, dy):
        h, G, U = pvq.pvq_fp8_gated(X, GATE, UP, out_dtype=torch.bfloat16, keep=True)
        return [h, G.codes, U.codes, pvq.pvq_fp8_product(X, GATE, torch.bfloat16), pvq.pvq_fp8_product(X, GATE, torch.float32),
                pvq.pvq_fp8_gated(X, GATE, UP, out_dtype=torch.bfloat16), pvq.pvq_fp8_input_grad(dy, down), pvq.pvq_fp8_input_grad(dy[:, :8999], pvq.Fp8Blocks(8999, 300, down.codes[:8999], down.exponents[:8999]))]
    sets = [inputs(1), inputs(2)]
    want = [[t.clone() for t in run(*i)] for i in sets]
    torch.cuda.synchronize()
    graphs = []
    for i in sets:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = run(*i)
        graphs.append((g, out))
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for turn in range(4):
        for (g, out), s in zip(graphs, streams):
            for t in out:
                t.fill_(1)
            s.wait_stream(torch.cuda.current_stream())
        for (g, out), s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        eager = run(*sets[turn % 2])
        torch.cuda.synchronize()
        for (g, out), w in zip(graphs, want):
            assert all(torch.equal(x, y) for x, y in zip(out, w)), turn
        assert all(torch.equal(x, y) for x, y in zip(eager, want[turn % 2]))
