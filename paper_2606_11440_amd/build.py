"""Build libinframind.so and libinframind_learn.so (all HIP sources, gfx950)
in-tree with hipcc."""
from __future__ import annotations

import concurrent.futures as cf
import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
BUILD = os.path.join(ROOT, "_build")
LIB = os.path.join(HERE, "libinframind.so")
SOURCES = ["route.hip", "schedule.hip", "rows.hip", "pool.hip"]
# the learner's operators: a library of their own
LEARN_LIB = os.path.join(HERE, "libinframind_learn.so")
LEARN_SOURCES = ["learn.hip", "learn_rows.hip", "learn_sums.hip", "learn_head.hip", "learn_adamw.hip",
                 "learn_experts.hip", "learn_router.hip", "learn_dispatch.hip", "learn_packed.hip"]
# measurement probe used by the benchmark only (not part of the tick's library)
PROBE_LIB = os.path.join(HERE, "libimprobe.so")
PROBE_SOURCES = ["peak_probe.hip"]

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
         # packed fp32 arithmetic stays off: plain fp32 code only
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-I", os.path.join(ROOT, "include"), "-I", CSRC]


def build(jobs: int = 6) -> str:
    """Compile every source and link the shared libraries; returns libinframind.so's path."""
    os.makedirs(BUILD, exist_ok=True)

    def compile_one(src):
        obj = os.path.join(BUILD, src + ".o")
        cmd = [HIPCC, *FLAGS, "-c", os.path.join(CSRC, src), "-o", obj]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"hipcc failed on {src}:\n{r.stderr}")
        return obj

    with cf.ThreadPoolExecutor(max_workers=jobs) as ex:
        objs = list(ex.map(compile_one, SOURCES + LEARN_SOURCES + PROBE_SOURCES))
    for lib, srcs in ((LIB, SOURCES), (LEARN_LIB, LEARN_SOURCES), (PROBE_LIB, PROBE_SOURCES)):
        tmp = lib + ".tmp"
        mine = [os.path.join(BUILD, s + ".o") for s in srcs]
        r = subprocess.run([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", tmp, *mine],
                           capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"link failed:\n{r.stderr}")
        os.replace(tmp, lib)
    return LIB


if __name__ == "__main__":
    print(build())
