"""Build the HIP library (libmpv.so) for gfx950, in-tree, with hipcc."""

import os
import shutil
import subprocess
import sys
import tempfile

PKG_DIR = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG_DIR)
SRC = os.path.join(PKG_DIR, "csrc", "mpv.hip")
LIB = os.path.join(PKG_DIR, "libmpv.so")

HIPCC_FLAGS = [
    "--offload-arch=gfx950",
    "-O3",
    "-std=c++17",
    "-fPIC",
    # no compiler-generated packed-fp32 instructions (v_pk_*_f32)
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wno-unused-command-line-argument",
]

# Translation units in link order, each with flags of its own.  The kernels of one unit are a code object of their own,
# so that where one unit's code lies does not depend on the others.
UNITS = {
    # the task loops are long and cold: loop-invariant constants hoisted out of them would be
    # held in registers across whole tasks and push the kept row pair into scratch memory
    "mpv.hip": ["-mllvm", "-disable-machine-licm"],
    # (so are the paths of a tile that few tiles take; -Winline-asm says that m0 is reserved wherever an instruction names it as written)
    "mpv_attention.hip": ["-mllvm", "-disable-machine-licm", "-Wno-inline-asm"],
    "mpv_prefix.hip": ["-mllvm", "-disable-machine-licm", "-Wno-inline-asm"],
    "mpv_behind.hip": ["-mllvm", "-disable-machine-licm", "-Wno-inline-asm"],
    "mpv_through.hip": ["-mllvm", "-disable-machine-licm", "-Wno-inline-asm"],
    "mpv_chains.hip": [],
    "mpv_cache.hip": [],
    "mpv_scores.hip": [],
    "mpv_evict.hip": [],
    "mpv_logprobs.hip": [],
}


def hipcc_path():
    return shutil.which("hipcc") or "/opt/rocm/bin/hipcc"


def build(verbose=True, extra_flags=()):
    """Compile csrc/*.hip into libmpv.so next to this file; always recompiles."""
    csrc = os.path.join(PKG_DIR, "csrc")
    with tempfile.TemporaryDirectory() as tmp:
        running, objects = [], []
        for unit, flags in UNITS.items():
            objects.append(os.path.join(tmp, unit + ".o"))
            cmd = [hipcc_path(), "-c", *HIPCC_FLAGS, *flags, *extra_flags, "-I", os.path.join(ROOT, "include"), "-I", csrc,
                   os.path.join(csrc, unit), "-o", objects[-1]]
            if verbose:
                print(" ".join(cmd), flush=True)
            running.append((cmd, subprocess.Popen(cmd)))
        codes = [(cmd, p.wait()) for cmd, p in running]
        for cmd, code in codes:
            if code:
                raise subprocess.CalledProcessError(code, cmd)
        cmd = [hipcc_path(), "--offload-arch=gfx950", "-shared", "-fPIC", *objects, "-o", LIB + ".tmp"]
        if verbose:
            print(" ".join(cmd), flush=True)
        subprocess.run(cmd, check=True)
    os.replace(LIB + ".tmp", LIB)
    return LIB


if __name__ == "__main__":
    build(extra_flags=sys.argv[1:])
