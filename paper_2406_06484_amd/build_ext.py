"""Builds libdeltanet_hip.so in-tree with hipcc for gfx950 (one object per .hip file, in parallel), and the Python module that calls its
attention operators with tensors (_attention.so, host code against torch's headers)."""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
OUT = os.path.join(HERE, "libdeltanet_hip.so")
BINDING = os.path.join(HERE, "_attention.so")
SOURCES = ["dn_api.hip", "dn_inst_f32.hip", "dn_inst_bf16.hip", "dn_inst_bf16_wide.hip", "dn_recurrent.hip", "dn_noalloc.hip", "dn_lds_probe.hip",
           "dn_attn_api.hip", "dn_norm_rope.hip", "dn_paged_attn.hip"]
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Wall", "-Wno-unused-function",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]


def _compile(src: str) -> str:
    obj = os.path.join(CSRC, "_build", os.path.splitext(src)[0] + ".o")
    os.makedirs(os.path.dirname(obj), exist_ok=True)
    # DELTANET_HIPCC_FLAGS: extra compiler flags
    cmd = ["hipcc"] + FLAGS + os.environ.get("DELTANET_HIPCC_FLAGS", "").split() + ["-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    err = "\n".join(l for l in r.stderr.splitlines() if "packed-fp32-ops" not in l)
    if r.returncode != 0:
        raise RuntimeError("hipcc failed on %s:\n%s" % (src, err))
    if err.strip():
        sys.stderr.write(err + "\n")
    return obj


def _compile_binding() -> None:
    """The module for calls with tensors.  It is left out, with a word on stderr, where there is no torch to serve or no host compiler; C callers need
    neither."""
    import sysconfig

    def left_out(why):
        if os.path.exists(BINDING):     # (none is better than one of other sources)
            os.remove(BINDING)
        sys.stderr.write("_attention.so is not built: no %s\n" % why)

    try:
        import torch
    except ImportError:
        return left_out("torch")
    root = os.path.dirname(torch.__file__)
    tmp = BINDING + ".tmp.%d" % os.getpid()
    cmd = ["g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-Wall", "-D_GLIBCXX_USE_CXX11_ABI=%d" % torch._C._GLIBCXX_USE_CXX11_ABI,
           "-isystem", os.path.join(root, "include"), "-isystem", os.path.join(root, "include", "torch", "csrc", "api", "include"),
           "-isystem", sysconfig.get_paths()["include"], os.path.join(CSRC, "dn_attention_binding.cpp"), "-o", tmp,
           "-L" + os.path.join(root, "lib"), "-Wl,-rpath," + os.path.join(root, "lib"), "-ltorch_python", "-ltorch_cpu", "-ltorch", "-lc10", "-ldl"]
    try:
        r = subprocess.run(cmd, capture_output=True, text=True)
    except FileNotFoundError:
        return left_out("g++")
    if r.returncode != 0:
        if os.path.exists(BINDING):
            os.remove(BINDING)
        raise RuntimeError("g++ failed on dn_attention_binding.cpp:\n" + r.stderr)
    if r.stderr.strip():
        sys.stderr.write(r.stderr)
    os.replace(tmp, BINDING)


def build(verbose: bool = True) -> str:
    with ThreadPoolExecutor(max_workers=len(SOURCES) + 1) as ex:
        binding = ex.submit(_compile_binding)
        objs = list(ex.map(_compile, SOURCES))
    tmp = OUT + ".tmp.%d" % os.getpid()
    subprocess.check_call(["hipcc", "--offload-arch=gfx950", "-shared", "-fPIC", "-o", tmp] + objs)
    os.replace(tmp, OUT)
    binding.result()    # (the library is there for C callers by now)
    if verbose:
        print("built", OUT)
    return OUT


if __name__ == "__main__":
    build()
