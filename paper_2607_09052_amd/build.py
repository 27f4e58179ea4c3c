"""Compile the COBS HIP library for gfx950 into this package directory.

    python -m paper_2607_09052_amd.build      (from the repository root)

Produces libcobs.so next to this file.  Packed-FP32 instructions are disabled
for every device compile.
"""
import glob
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
LIB = os.path.join(HERE, "libcobs.so")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++20", "-fPIC",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function",
]
DIRS = ("csrc", "csrc_cache", "csrc_tokens")
OBJ_DIR = os.path.join(HERE, "_build")


def sources():
    """The decode path's translation units, then those of the operators around it (their names differ)."""
    return [s for d in DIRS for s in sorted(glob.glob(os.path.join(HERE, d, "*.hip")))]


def _run(cmd):
    res = subprocess.run(cmd, capture_output=True, text=True)
    errs = "\n".join(l for l in (res.stdout + res.stderr).splitlines()
                     if "packed-fp32-ops" not in l and "target-feature" not in l)
    return res.returncode, errs


def build(verbose=False, jobs=None):
    """Compile every translation unit (in parallel), then link libcobs.so."""
    from concurrent.futures import ThreadPoolExecutor
    os.makedirs(OBJ_DIR, exist_ok=True)
    inc = ["-I", os.path.join(ROOT, "include")] + [x for d in DIRS for x in ("-I", os.path.join(HERE, d))]
    srcs = sources()
    objs = [os.path.join(OBJ_DIR, os.path.basename(s)[:-4] + ".o") for s in srcs]
    cmds = [[HIPCC, *FLAGS, *inc, "-c", s, "-o", o] for s, o in zip(srcs, objs)]
    jobs = jobs or min(len(cmds), int(os.environ.get("MAX_JOBS", os.cpu_count() or 4)), 8)
    with ThreadPoolExecutor(max_workers=max(1, jobs)) as ex:
        results = list(ex.map(_run, cmds))
    for cmd, (rc, errs) in zip(cmds, results):
        if verbose:
            print(" ".join(cmd), flush=True)
        if rc != 0:
            raise RuntimeError(f"hipcc failed ({rc}) on {cmd[-3]}:\n{errs}")
        if verbose and errs.strip():
            print(errs)
    tmp = LIB + ".tmp"
    rc, errs = _run([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", *objs, "-o", tmp])
    if rc != 0:
        raise RuntimeError(f"link failed ({rc}):\n{errs}")
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
