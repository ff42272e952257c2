"""Build libkvprm.so in-tree for gfx950 with hipcc."""
import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
LIB = os.path.join(HERE, "libkvprm.so")
SOURCES = ["kvprm_api.hip", "kvprm_kernels.hip", "kvprm_mfma.hip", "kvprm_attn.hip", "kvprm_f32.hip",
           "kvprm_grad.hip", "kvprm_cache.hip", "kvprm_tree.hip"]
FLAGS = ["--offload-arch=gfx950", "-O3", "-fPIC", "-shared", "-std=c++17",
         # packed fp32 instructions are disabled on purpose for this target
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-Wno-unused-command-line-argument"]


def build(verbose: bool = False) -> str:
    src = [os.path.join(HERE, "csrc", s) for s in SOURCES]
    cmd = [HIPCC, *FLAGS, "-I", os.path.join(ROOT, "include"), *src, "-o", LIB]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("libkvprm build failed:\n" + " ".join(cmd) + "\n" + r.stdout + r.stderr)
    if verbose and r.stderr.strip():
        print(r.stderr)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
