"""Compile the HIP attention library for gfx950 into an in-tree shared object."""
from __future__ import annotations

import os
import shutil
import subprocess
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB_PATH = os.path.join(HERE, "libvitattn.so")
SOURCES = ["vitattn_api.hip", "vitattn_fwd.hip", "vitattn_bwd.hip", "vitattn_merge.hip", "vitattn_ulysses.hip", "vitattn_agg.hip",
           "vitattn_block_api.hip", "vitattn_rows_api.hip", "vitattn_norm.hip", "vitattn_rms.hip", "vitattn_rms_bwd.hip", "vitattn_dropout.hip", "vitattn_rotary.hip", "vitattn_diff_fwd.hip", "vitattn_diff_bwd.hip",
           "vitattn_sparse_api.hip", "vitattn_select.hip", "vitattn_sparse_fwd.hip", "vitattn_sparse_bwd.hip",
           "vitattn_sparse_dkdv.hip", "vitattn_sparse_dq.hip"]
ARCH = "gfx950"

HIP_FLAGS = [
    f"--offload-arch={ARCH}",
    "-O3",
    "-std=c++17",
    "-fPIC",
    "-Wall", "-Wextra",
    # packed fp32 VALU forms stay disabled on this target
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    # keep matrix-core accumulators in VGPR form: otherwise the allocator
    # parks loop-carried accumulators in AGPRs and copies them every trip
    "-mllvm", "-amdgpu-mfma-vgpr-form=1",
]


def hipcc() -> str:
    for cand in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", shutil.which("hipcc")):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("hipcc not found: cannot build the gfx950 attention library")


# Debug variant for the tests: every kernel first fills its LDS with NaN bytes,
# so a read of LDS that nothing wrote shows up as NaN (never used by the
# package itself; tests load it explicitly).
LDS_POISON_LIB_PATH = os.path.join(HERE, "libvitattn_ldspoison.so")


def _run(cmds, verbose):
    """Runs the commands, as many at a time as there are CPUs for; raises with
    the output of those that failed."""
    def one(cmd):
        if verbose:
            print(" ".join(cmd), flush=True)
        return cmd, subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.PIPE, text=True)

    jobs = min(len(os.sched_getaffinity(0)), int(os.environ.get("MAX_JOBS", "16")))
    with ThreadPoolExecutor(max(1, jobs)) as ex:
        failed = [f"{c[-1]}: hipcc failed ({p.returncode}):\n{p.stdout}\n{p.stderr}" for c, p in ex.map(one, cmds)
                  if p.returncode != 0]
    if failed:
        raise RuntimeError("\n".join(failed))


def build(verbose: bool = False, lds_poison: bool = True) -> str:
    """Always recompiles; writes LIB_PATH (and, with lds_poison, the LDS-poison
    debug variant, compiled alongside) atomically and returns LIB_PATH. Each
    source is compiled on its own, side by side."""
    libs = [(LIB_PATH, ())]
    if lds_poison:
        libs.append((LDS_POISON_LIB_PATH, ("-DVITATTN_DEBUG_LDS_POISON",)))
    with tempfile.TemporaryDirectory() as tmp:
        compiles, links = [], []
        for n, (path, extra) in enumerate(libs):
            objects = [os.path.join(tmp, f"{n}_{s}.o") for s in SOURCES]
            compiles += [[hipcc(), *HIP_FLAGS, *extra, "-c", "-o", o, os.path.join(CSRC, s)]
                         for s, o in zip(SOURCES, objects)]
            links.append([hipcc(), f"--offload-arch={ARCH}", "-fPIC", "-shared", "-o", path + f".tmp{os.getpid()}", *objects])
        # the longest compilations first
        compiles.sort(key=lambda c: -os.path.getsize(c[-1]))
        _run(compiles, verbose)
        _run(links, verbose)
    for path, _ in libs:
        os.replace(path + f".tmp{os.getpid()}", path)
    return LIB_PATH


if __name__ == "__main__":
    print(build(verbose=True))
