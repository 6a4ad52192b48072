"""Build libcrisp.so for gfx950 with hipcc (in-tree, next to this file)."""
import os
import subprocess
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libcrisp.so")
OBJDIR = os.path.join(HERE, "_build")

SOURCES = ["spmm_nm_2_4.hip", "spmm_nm_4_8.hip", "spmm_nm_3_4.hip", "spmm_nm_4_4.hip", "spmm_nm_8_8.hip", "spmm_nm_1_4.hip",
           "spmm_nm_2_8.hip", "spmm_nm_1_8.hip", "spmm_lds.hip", "spmm_kernels.hip", "crisp_api.hip", "select_kernels.hip",
           "pack_kernels.hip", "im2col_kernels.hip", "budget_kernels.hip", "fp8_quant.hip", "fp8_product.hip", "fp8_tiled.hip", "fp8_split.hip", "fp8_api.hip",
           "adamw.hip"]

FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-fvisibility=hidden", "-ffp-contract=off",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-I" + os.path.join(ROOT, "include"), "-I" + CSRC, "-Wall", "-Wno-unused-command-line-argument"]


def _compile(src: str) -> str:
    obj = os.path.join(OBJDIR, src.replace(".hip", ".o"))
    cmd = ["hipcc"] + FLAGS + ["-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    err = "\n".join(l for l in r.stderr.splitlines() if "not a recognized feature" not in l)
    if r.returncode != 0:
        raise RuntimeError("hipcc failed for %s:\n%s" % (src, err))
    if err.strip():
        print(err)
    return obj


def build(jobs: int = 8) -> str:
    os.makedirs(OBJDIR, exist_ok=True)
    with ThreadPoolExecutor(max_workers=jobs) as ex:
        objs = list(ex.map(_compile, SOURCES))
    cmd = ["hipcc", "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB] + objs
    subprocess.run(cmd, check=True)
    return LIB


if __name__ == "__main__":
    print(build())
