"""The tiles of 8-bit blocks keep their sums in accumulation registers that assembly statements write: the compiler knows of no wait
between these and what reads them.  So it must not move sums about, read them at places of its own or keep registers in memory."""
import os
import re
import subprocess

import pytest

from paper_2410_16926_amd import build

CSRC = os.path.join(os.path.dirname(os.path.abspath(build.__file__)), "csrc")
KERNEL = re.compile(r"^(_ZN\S*?\d(?:wide_tile_kernel|tile_kernel|grad_kernel)\S*):", re.M)


@pytest.mark.parametrize("name,kernels", [("pvq_fp8_grad.hip", 4), ("pvq_fp8_product.hip", 5)])
def test_sums_stay_where_they_are(name, kernels, tmp_path):
    out = str(tmp_path / "kernels.s")
    flags = [f for f in build.HIPCC_FLAGS if f != "-shared"]
    include = os.path.join(os.path.dirname(os.path.dirname(CSRC)), "include")
    subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), *flags, "-x", "hip", f"-I{include}", f"-I{CSRC}", "--cuda-device-only", "-S",
                    os.path.join(CSRC, name), "-o", out], check=True, capture_output=True)
    with open(out) as f:
        text = f.read()
    found = list(KERNEL.finditer(text))
    assert len(found) == kernels
    for m in found:
        body = text[m.end():text.index(".end_amdhsa_kernel", m.end())]
        lines = [line.strip() for line in body.split("\n")]
        assert not any(line.startswith(("scratch_", "v_accvgpr_mov")) for line in lines), m.group(1)
        # every read is one of ours, behind the wait: each sum once
        reads = [i for i, line in enumerate(lines) if line.startswith("v_accvgpr_read")]
        assert len(reads) == (128 if "ELi4E" in m.group(1) else 256), m.group(1)
        assert all(lines[i - 1] == ";;#ASMSTART" for i in reads), m.group(1)
        # nothing but zeros in front of the steps is written to them besides
        last = max(i for i, line in enumerate(lines) if line.startswith("v_mfma"))
        writes = [line for line in lines[:last] if line.startswith("v_accvgpr_write")]
        assert all(re.search(r", 0$", line) for line in writes), m.group(1)
