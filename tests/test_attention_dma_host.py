"""The paged attention's transfers to the LDS are written in inline asm, as the chunk kernel's: the same distances, read from the compiled code (no GPU needed)."""
import os
import re
import shutil
import subprocess

import pytest

from tests.test_dma_hazards_host import CSRC, _instructions, _read_too_early


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="needs hipcc")
def test_transfers_to_the_lds():
    asm = subprocess.run(["hipcc", "--offload-arch=gfx950", "-O3", "-std=c++17", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-w",
                          "--offload-device-only", "-S", os.path.join(CSRC, "dn_paged_attn.hip"), "-o", "-"], check=True, capture_output=True, text=True).stdout
    kernels = re.findall(r"^(_ZN2dn11k_attn_(?:wide|both)IDF16b\w+):(.*?)s_endpgm", asm, re.M | re.S)
    assert len(kernels) == 6
    for name, body in kernels:
        ops = list(_instructions(body))
        moves = [i for i, (op, words) in enumerate(ops) if op.startswith("buffer_load") and "lds" in words]
        assert moves, name
        assert not _read_too_early(body), name
        for i in moves:     # M0 is written right in front of its own transfer, one wait state at least between them, and by nothing else
            assert [op for op, _ in ops[i - 2:i]] == ["s_mov_b32", "s_nop"] and ops[i - 2][1][0] == "m0", name
        assert sum("m0" in words for _, words in ops) == len(moves), name
