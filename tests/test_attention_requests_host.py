"""What the attention of few rows asks the cache for goes through descriptors, whose range is nothing behind a wave's last step: read from the compiled code (no GPU needed)."""
import os
import re
import shutil
import subprocess

import pytest

from tests.test_dma_hazards_host import CSRC, _instructions


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="needs hipcc")
def test_requests_of_a_further_step_have_a_range():
    asm = subprocess.run(["hipcc", "--offload-arch=gfx950", "-O3", "-std=c++17", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-w",
                          "--offload-device-only", "-S", os.path.join(CSRC, "dn_paged_attn.hip"), "-o", "-"], check=True, capture_output=True, text=True).stdout
    kernels = re.findall(r"^(_ZN2dn10k_attn_few\w+):(.*?)\.Lfunc_end", asm, re.M | re.S)
    assert len(kernels) == 20
    for name, body in kernels:
        ops = [op for op, _ in _instructions(body)]
        products = [i for i, op in enumerate(ops) if op.startswith("v_mfma")]
        loads = [op for op in ops[products[0]:products[-1] + 1] if re.match(r"(global|flat|buffer)_load_dwordx[24]", op)]
        assert loads and all(op.startswith("buffer") for op in loads), (name, loads)     # (single words: the page table's entries)
