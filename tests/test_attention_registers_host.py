"""No kernel of the attention operators keeps registers in scratch memory.  A spilled four-register operand has been compiled here with one of its
registers never brought back (saved to an accumulator register that nothing reads again), which shows as wrong numbers and only where that kernel
runs; a kernel that does not spill cannot meet it.  Read from the compiler's report (no GPU needed)."""
import os
import re
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2406_06484_amd", "csrc")


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="needs hipcc")
@pytest.mark.parametrize("source,kernels", [("dn_paged_attn.hip", 42), ("dn_norm_rope.hip", 76)])
def test_no_spilled_registers(source, kernels, tmp_path):
    r = subprocess.run(["hipcc", "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-w",
                        "--offload-device-only", "-Rpass-analysis=kernel-resource-usage", "-c", os.path.join(CSRC, source), "-o", str(tmp_path / "x.o")],
                       check=True, capture_output=True, text=True)
    names = re.findall(r"Function Name: (\S+)", r.stderr)
    scratch, spilled = (list(map(int, re.findall(p, r.stderr))) for p in (r"ScratchSize \[bytes/lane\]: (\d+)", r"VGPRs Spill: (\d+)"))
    assert len(names) == len(scratch) == len(spilled) and len(names) >= kernels
    assert not [(n, a, b) for n, a, b in zip(names, scratch, spilled) if a or b]
