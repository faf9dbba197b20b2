"""Workspaces of the gated block are what include/pvq.h says: nothing where one kernel has it all, else the float32 sums of G and U for each part."""
import ctypes as C

import pytest

import paper_2410_16926_amd as pvq

F32, F16, BF16 = 0, 1, 2


@pytest.mark.parametrize("m,n,k", [(1, 28672, 8192), (32, 14336, 4096), (33, 1500, 1500), (64, 1500, 1500), (70, 300, 9000), (517, 14336, 4096), (132, 5637, 4311), (1316, 4457, 66),
                                   (2048, 28672, 8192), (1, 1, 1)])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_the_gated_block_passes_sums_through_the_workspace(m, n, k, dtype):
    def sums(call, t):
        kind, parts = pvq.pvq_fp8_plan(call, m, n, k, t)
        joined = kind != "rows" and (parts > 1 or (kind == "tiles_64" and call != "gated"))
        return 8 * m * n * parts if joined else 0
    got = C.c_size_t()
    for to_blocks, calls in ((0, ("gated",)), (1, ("gated_to_blocks", "gated_kept"))):
        assert pvq.lib().pvq_fp8_gated_work_bytes(m, n, k, dtype, to_blocks, C.byref(got)) == 0
        # either instruction: that of float32 results and that of the others
        assert got.value == max(sums(c, t) for c in calls for t in (F32, BF16))


@pytest.mark.parametrize("m,n,k", [(1, 1, 1), (517, 14336, 4096), (65, 4609, 1625), (2048, 14336, 4096)])
def test_the_backward_pass_has_slopes_in_two_pieces_and_the_longest_split(m, n, k):
    slopes = 2 * 2 * m * -(-n // 64) * 64 * 2
    sums = 0
    for t in (F32, BF16):
        for call, values in (("gated_input_grad", m * k), ("gated_weight_grads", 2 * n * k)):
            parts = pvq.pvq_fp8_plan(call, m, n, k, t)[1]
            sums = max(sums, 4 * parts * values if parts > 1 else 0)
    got = C.c_size_t()
    assert pvq.lib().pvq_fp8_gated_backward_work_bytes(m, n, k, C.byref(got)) == 0
    assert got.value == slopes + sums
