"""Builds libfmtc.so (the C-ABI library) in-tree with hipcc for gfx950."""
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libfmtc.so")
SOURCES = ["fmtc_api.hip", "fmtc_encode_kernels.hip", "fmtc_coder_kernels.hip", "fmtc_decode_kernels.hip",
           "fmtc_fit_kernels.hip", "fmtc_int8_kernels.hip", "fmtc_profile.hip", "fmtc_block_api.hip",
           "fmtc_quantize_f8_kernels.hip", "fmtc_matmul_f8_kernels.hip", "fmtc_norm_kernels.hip",
           "fmtc_matmul_i8_kernels.hip", "fmtc_group_norm_kernels.hip", "fmtc_clip_kernels.hip"]
FLAGS = ["-O3", "-std=c++17", "--offload-arch=gfx950", "-fPIC", "-Wall",
         # packed fp32 VALU forms are kept off on purpose
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-I" + os.path.join(ROOT, "include"), "-I" + CSRC]


def build(verbose=False):
    """Compile every source and link the shared library.  Always recompiles."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    objs = []
    procs = []
    for src in SOURCES:
        obj = os.path.join(CSRC, src.replace(".hip", ".o"))
        objs.append(obj)
        cmd = [hipcc] + FLAGS + ["-c", os.path.join(CSRC, src), "-o", obj]
        if verbose:
            print(" ".join(cmd), flush=True)
        procs.append((src, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    for src, pr in procs:
        out, _ = pr.communicate()
        out = "\n".join(l for l in out.splitlines() if "packed-fp32-ops" not in l)
        if pr.returncode != 0:
            raise RuntimeError(f"hipcc failed on {src}:\n{out}")
        if out.strip() and verbose:
            print(out)
    subprocess.run([hipcc, "-shared", "--offload-arch=gfx950", "-o", LIB] + objs, check=True)
    return LIB


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
