"""The attention operators' C ABI (argument validation, sizes, dispatch) built for the CPU with AddressSanitizer and UndefinedBehaviorSanitizer: host
code only, against stand-ins for the launches (tests/sanitize/)."""
import os
import shutil
import subprocess

import pytest

from tests.test_sanitizers_host import ROOT, SAN, _run


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="hipcc not on PATH")
def test_attention_host_layer_under_address_and_undefined_behaviour_sanitizers(tmp_path):
    exe = str(tmp_path / "attn_san")
    cmd = ["hipcc", "--offload-host-only", "-x", "hip", "-O1", "-g", "-std=c++17",
           "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fno-sanitize-recover=all",
           os.path.join(ROOT, "paper_2406_06484_amd", "csrc", "dn_attn_api.hip"), os.path.join(SAN, "attn_stubs.cpp"),
           os.path.join(SAN, "attn_main.cpp"), "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stderr[-3000:]
    assert "attention host layer under sanitizers: ok" in _run(exe)
