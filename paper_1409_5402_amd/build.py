"""Compiles the HIP library for gfx950 in-tree (hipcc cross-compiles without a GPU)."""
from __future__ import annotations

import os
import subprocess
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
SRC = [os.path.join(HERE, "csrc", name) for name in ("same_lda.hip", "word_table.hip", "embed_grad.hip", "embed_grad_dropout_float.hip",
                                                     "embed_grad_dropout_bfloat.hip", "embed_grad_dropout_half.hip", "word_rows.hip",
                                                     "group_table.hip")]
LIB = os.path.join(HERE, "libsame_lda.so")

# -ffp-contract=off: every binary32 step of the draw is rounded once (no fused multiply-add);
# packed-fp32 instructions are disabled for the device pass.
FLAGS = ["-O3", "--offload-arch=gfx950", "-std=c++17", "-ffp-contract=off",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-fPIC", "-Wall", "-Wextra", "-Wno-unused-value"]


STATS_LIB = os.path.join(HERE, "libsame_lda_stats.so")


def build(verbose: bool = False, stats: bool = False) -> str:
    """stats=True builds a second library whose draw kernel counts its own events (steps, trips, pmf terms,
    shared passes) into a device buffer given through same_lda_stats_buffer: for `bench.py --mode stats` only."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    lib = STATS_LIB if stats else LIB
    flags = [*FLAGS, *(["-DSAME_STATS"] if stats else [])]
    with tempfile.TemporaryDirectory() as where:                 # the sources side by side, then one library
        objects = [os.path.join(where, os.path.basename(src) + ".o") for src in SRC]
        compiles = [[hipcc, *flags, "-c", src, "-o", obj] for src, obj in zip(SRC, objects)]
        started = [(cmd, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)) for cmd in compiles]
        results = [(cmd, run.communicate()[0], run.returncode) for cmd, run in started]
        if not any(rc for _, _, rc in results):
            link = [hipcc, "--offload-arch=gfx950", "-fPIC", "-shared", "-o", lib, *objects]
            run = subprocess.run(link, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
            results.append((link, run.stdout, run.returncode))
    for cmd, text, rc in results:
        if verbose or rc != 0:
            print(" ".join(cmd))
            print(text)
    if any(rc for _, _, rc in results):
        raise RuntimeError("hipcc failed building the library")
    return lib


if __name__ == "__main__":
    import sys
    print(build(verbose=True, stats="--stats" in sys.argv))
