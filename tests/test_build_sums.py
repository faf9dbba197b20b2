"""No library is linked of code in which the compiler has touched the sums that assembly statements form.  Nothing is compiled for a GPU here."""
import os
import sys

import pytest

from paper_2410_16926_amd import build

GOOD = """
_ZN12_GLOBAL__N_111grad_kernelILi1ELi8EEEvN3abc: ; @kernel
	v_accvgpr_write_b32 a0, 0
	v_add_u32_e32 v9, v1, v2
.LBB0_1:                                ; =>loop
	v_mov_b32_e32 v20, 0
	;;#ASMSTART
	v_mfma_f32_16x16x32_bf16 a[0:3], v[4:7], v[10:13], a[0:3]
	;;#ASMEND
	v_cvt_pk_bf16_f32 v4, v20, v21
	s_nop 1
	;;#ASMSTART
	v_mfma_f32_16x16x32_bf16 a[0:3], v[4:7], v[10:13], a[0:3]
	;;#ASMEND
	v_mov_b32_e32 v10, v20
	s_add_i32 s0, s0, 1
	s_cbranch_scc1 .LBB0_1
	;;#ASMSTART
	v_accvgpr_read_b32 v30, a0
	;;#ASMEND
	s_endpgm
	.end_amdhsa_kernel
"""


def test_code_that_leaves_the_sums_alone():
    assert build.disturbed_sums(GOOD) == []


@pytest.mark.parametrize("old,new,line", [
    ("	s_nop 1\n", "", "v_mfma"),                                                     # an operand written just in front
    ("	s_nop 1\n", "	s_nop 0\n", "v_mfma"),
    ("	s_nop 1\n", "	s_nop 0\n	ds_read_b32 v40, v41\n", None),                     # (two others in between will do)
    ("	s_add_i32 s0, s0, 1\n	s_cbranch", "	s_cbranch", None),                       # by way of the jump back: the jump and a move between
    ("	v_mov_b32_e32 v20, 0\n", "", None),                                           # (an addition and the jump)
    ("	v_mov_b32_e32 v20, 0\n", "	v_mov_b32_e32 v13, 0\n", "v_mfma"),
    ("	v_mov_b32_e32 v20, 0\n", "	scratch_load_dword v20, off, s4\n", "scratch_load"),
    ("	v_mov_b32_e32 v20, 0\n", "	v_accvgpr_mov_b32 a4, a0\n", "v_accvgpr_mov"),
    ("	v_mov_b32_e32 v20, 0\n", "	v_accvgpr_read_b32 v20, a0\n", "v_accvgpr_read"),
    ("	v_mov_b32_e32 v20, 0\n", "	v_accvgpr_write_b32 a0, v3\n", "v_accvgpr_write"),
    ("grad_kernel", "other_kernel", "no kernels"),
])
def test_code_that_does_not(old, new, line):
    assert GOOD.count(old) == 1
    wrong = build.disturbed_sums(GOOD.replace(old, new))
    assert wrong == [] if line is None else wrong and all(line in w for w in wrong)


def test_without_a_wait_on_the_way_back():
    text = GOOD.replace("	s_add_i32 s0, s0, 1\n", "").replace("	v_mov_b32_e32 v20, 0\n", "")
    wrong = build.disturbed_sums(text)
    assert len(wrong) == 1 and "v_mfma" in wrong[0]


def compiler(tmp_path, text):
    """A stand-in for the compiler that writes an object, and a listing beside it where it is asked for one."""
    path = tmp_path / "compiler.py"
    path.write_text(f"""#!{sys.executable}
import sys
out = sys.argv[sys.argv.index("-o") + 1]
open(out, "w").write("object")
if "{build.KEEP_LISTING}" in sys.argv:
    stem = out[:out.index(".hip")]
    open(stem + "-hip-amdgcn-amd-amdhsa-gfx950.s", "w").write({text!r})
    open(stem + "-host-x86_64-unknown-linux-gnu.s", "w").write("")
    open(stem + ".hip-hip-amdgcn-amd-amdhsa.hipfb", "w").write("")
""")
    path.chmod(0o755)
    return str(path)


@pytest.mark.parametrize("text,good", [(GOOD, True), (GOOD.replace("	s_nop 1\n", ""), False), ("", False)])
def test_nothing_is_linked_of_such_code(tmp_path, monkeypatch, text, good):
    monkeypatch.setenv("HIPCC", compiler(tmp_path, text))
    monkeypatch.setattr(build, "_HERE", str(tmp_path))
    monkeypatch.setattr(build, "LIB_PATH", str(tmp_path / "libpvq.so"))
    if good:
        build.build(binding=False)
        assert os.path.exists(tmp_path / "libpvq.so")
    else:
        with pytest.raises(RuntimeError, match="could form wrong sums"):
            build.build(binding=False)
        assert not os.path.exists(tmp_path / "libpvq.so")
    left = sorted(os.listdir(tmp_path / "_build"))
    assert all(name.endswith(".o") for name in left)
    assert all((name + ".o" in left) == good for name in build.SUMS_IN_ASSEMBLY)
