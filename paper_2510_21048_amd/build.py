"""Build libxmem_replay.so (replay and trace preparation) and libxmem_ops.so (the training operators)
in-tree with hipcc for gfx950."""
from __future__ import annotations

import os
import subprocess
from pathlib import Path

PKG = Path(__file__).resolve().parent
ROOT = PKG.parent
SRCS = [PKG / "csrc" / "xmem_replay.hip", PKG / "csrc" / "xmem_prep.hip"]
LIB = PKG / "libxmem_replay.so"
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared",
    # no packed fp32 instructions anywhere (none are needed: the path is integer-only)
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    # the row tables order their integer keys as doubles, none of them a NaN: min and max need no quieting
    "-fno-honor-nans",
    # the event loops branch on wave-uniform values only: left unstructured, both sides of a branch update
    # the table's registers in place (structured, each side keeps a copy: 1.7x the registers, and spills
    # in the loops; as it is, k_chunk_sched<false> and k_rs_scatter spill a few registers a tile, none
    # of them between two events, which tests/test_abi_host.py holds them to)
    "-mllvm", "-structurizecfg-skip-uniform-regions=1",
]


# The operators are a library of their own: they compute on floating numbers, NaN among them, which the
# replay's flags rule out.
OPS_SRCS = sorted((PKG / "csrc" / "ops").glob("*.hip"))
OPS_LIB = PKG / "libxmem_ops.so"
OPS_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared",
    # no packed fp32 instructions
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
]


def _start(flags, srcs, out: Path):
    return subprocess.Popen([HIPCC, *flags, f"-I{ROOT / 'include'}", *map(str, srcs), "-o", str(out)],
                            stderr=subprocess.PIPE)


def _finish(proc, tmp: Path, lib: Path) -> None:
    err = proc.communicate()[1]
    if proc.returncode:
        raise subprocess.CalledProcessError(proc.returncode, proc.args, stderr=err)
    os.replace(tmp, lib)


def build() -> Path:
    """Compile both libraries every time it is called, side by side (under a minute)."""
    started = []
    for flags, srcs, lib in ((FLAGS, SRCS, LIB), (OPS_FLAGS, OPS_SRCS, OPS_LIB)):
        tmp = lib.with_suffix(".so.tmp")
        started.append((_start(flags, srcs, tmp), tmp, lib))
    for proc, tmp, lib in started:
        _finish(proc, tmp, lib)
    return LIB


if __name__ == "__main__":
    print(build())
