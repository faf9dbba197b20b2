"""Which tiles the calls on 8-bit blocks take, asked for without launching anything."""
import ctypes as C

import pytest

import paper_2410_16926_amd as pvq
from tests import fp8_tiles

INVALID, UNSUPPORTED = -1, -2


@pytest.mark.parametrize("case", fp8_tiles.KINDS)
def test_the_shapes_of_the_tests_are_taken_by_the_tiles_that_they_are_for(case):
    call, dtype, *shape = case
    kind, parts = pvq.pvq_fp8_plan(call, *shape, dtype)
    assert (kind, parts > 1) == fp8_tiles.KINDS[case]


def test_every_kind_of_large_tile_is_among_them():
    of = {}
    for (call, _, *_), kind in fp8_tiles.KINDS.items():
        of.setdefault(call, set()).add(kind)
    both = {(k, s) for k in ("tiles_128", "tiles_256") for s in (False, True)}
    for call in ("input_grad", "weight_grad", "gated_input_grad", "gated_weight_grads"):
        assert of[call] == both
    eight = {("tiles_8bit", False), ("tiles_8bit", True)}
    whole = {("tiles_256", False), ("tiles_256", True)}
    assert of["product"] == both | eight and of["gated"] == whole | eight and of["gated_to_blocks"] == eight and of["gated_kept"] == whole


def test_few_rows_and_small_products():
    for n, k in ((1, 1), (1024, 8192), (28672, 8192)):
        assert pvq.pvq_fp8_plan("product", 1, n, k) == pvq.pvq_fp8_plan("product", 32, n, k) == ("rows", 1)
        assert pvq.pvq_fp8_plan("gated", 32, n, k) == ("rows", 1)
        assert pvq.pvq_fp8_plan("product", 33, n, k)[0] != "rows" and pvq.pvq_fp8_plan("gated", 33, n, k)[0] != "rows"
        for call in ("gated_to_blocks", "gated_kept"):
            assert pvq.pvq_fp8_plan(call, 32, n, k)[0] != "rows"
    assert pvq.pvq_fp8_plan("product", 64, 1500, 1500)[0] == "tiles_64"
    # what holds no 8-bit sums whatever the shape
    for m in (33, 512, 8192):
        for call, dtype in (("product", 0), ("gated", 0), ("gated_kept", 0), ("gated_kept", 1), ("gated_kept", 2)):
            assert pvq.pvq_fp8_plan(call, m, 8192, 8192, dtype)[0] != "tiles_8bit"


def test_the_plan_refuses():
    L = pvq.lib()
    a, b = C.c_int(), C.c_int()
    assert L.pvq_fp8_plan(0, 2, 3, 4, 0, C.byref(a), C.byref(b)) == 0
    for args in ((8, 2, 3, 4, 0), (-1, 2, 3, 4, 0), (0, 0, 3, 4, 0), (0, 2, 0, 4, 0), (0, 2, 3, 0, 0), (0, -2, 3, 4, 0), (0, 2, 3, 4, 3)):
        assert L.pvq_fp8_plan(*args, C.byref(a), C.byref(b)) == INVALID
    assert L.pvq_fp8_plan(0, 2, 3, 4, 0, None, C.byref(b)) == L.pvq_fp8_plan(0, 2, 3, 4, 0, C.byref(a), None) == INVALID
    assert L.pvq_fp8_plan(0, 2, 3, (1 << 22) + 1, 0, C.byref(a), C.byref(b)) == L.pvq_fp8_plan(1, 2, (1 << 22) + 1, 4, 0, C.byref(a), C.byref(b)) == UNSUPPORTED
    assert L.pvq_fp8_plan(0, 2, (1 << 22) + 1, 4, 0, C.byref(a), C.byref(b)) == 0           # (a product's rows of weights)
