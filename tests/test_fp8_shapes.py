"""Shapes of 8-bit blocks that do not belong together although their planes, whole blocks of 128 columns, have the same size.  No GPU."""
import pytest

import paper_2410_16926_amd as pvq

torch = pytest.importorskip("torch")


def blocks(rows, cols):
    per = -(-cols // 128)
    return pvq.Fp8Blocks(rows, cols, torch.zeros(rows, 128 * per, dtype=torch.uint8), torch.zeros(rows, 4 * -(-per // 4), dtype=torch.uint8))


def test_the_backward_pass_refuses_kept_products_of_another_shape():
    m, n, k = 3, 300, 200
    X, gate, up, right = blocks(m, k), blocks(n, k), blocks(n, k), blocks(m, n)
    dh = torch.zeros(m, n, dtype=torch.bfloat16)
    for wrong in (blocks(m, n - 1), blocks(m, n + 1), blocks(m, 257), blocks(m, 384), blocks(m + 1, n), blocks(m - 1, n)):
        for kept in ((wrong, right), (right, wrong), (wrong, wrong)):
            for wanted in ((True, True), (True, False), (False, False)):
                with pytest.raises(ValueError, match="kept products"):
                    pvq.pvq_fp8_gated_backward(dh, X, gate, up, *kept, "silu", None, *wanted)
    with pytest.raises(ValueError, match="hidden units"):
        pvq.pvq_fp8_gated_backward(dh, X, gate, blocks(n + 1, k), right, right)
    with pytest.raises(ValueError, match="GPU"):                 # the right ones come as far as the tensors
        pvq.pvq_fp8_gated_backward(dh, X, gate, up, right, right)
