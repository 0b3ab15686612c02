"""Builds libctc_mi355x.so for gfx950 with hipcc, and the CPython modules that call it, in-tree next to this file.

    python -m paper_1512_02595_amd.build

hipcc cross-compiles without a GPU.  Packed-fp32 code generation is switched off
for all device code.  The CTC path and the output layer's calls are compiled apart
(the former takes it that no NaN arises) and linked into one library.
"""
from __future__ import annotations

import os
import subprocess
import sys
import sysconfig
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libctc_mi355x.so")
SOURCES = ["ctc_kernels.hip", "ctc_api.cpp"]
LAYER_SOURCES = ["layer_kernels.hip", "layer_api.cpp"]
BINDING = os.path.join(HERE, "_binding.so")
LAYER_BINDING = os.path.join(HERE, "_layer_binding.so")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


def _hipcc(more: list[str], out: str) -> list[str]:
    return [HIPCC, "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
            "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
            "-Wall", "-Wextra", "-Wno-unused-command-line-argument",
            *os.environ.get("CTC_EXTRA_HIPCC_FLAGS", "").split(),
            "-I", os.path.join(ROOT, "include"), "-I", CSRC, *more, "-o", out]


def object_command(source: str, out: str) -> list[str]:
    """One source to an object.  No NaN ever enters the CTC path's arithmetic (log 0 is a finite sentinel): that lets
    max/min skip the quieting of their operands.  The output layer's calls pass NaNs on."""
    flags = ["-fno-honor-nans"] if source in SOURCES else []
    return _hipcc([*flags, "-x", "hip", "-c", os.path.join(CSRC, source)], out)


def link_command(objects: list[str], out: str = LIB) -> list[str]:
    return _hipcc(["-shared", *objects], out)


def binding_command(source: str, out: str) -> list[str]:
    """Host code only: the interpreter's symbols are resolved when it loads the module."""
    return [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall", "-Wextra",
            "-Wno-missing-field-initializers",
            "-I", sysconfig.get_paths()["include"], "-I", os.path.join(ROOT, "include"),
            os.path.join(CSRC, source), "-o", out]


def _compile(cmd: list[str], tmp: str, target: str, verbose: bool) -> None:
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        sys.stderr.write(res.stdout + res.stderr)
        raise RuntimeError(f"{cmd[0]} failed building {os.path.basename(target)}")
    if verbose and res.stderr.strip():
        sys.stderr.write(res.stderr)
    os.replace(tmp, target)


def build(verbose: bool = False) -> str:
    for target, source in ((BINDING, "binding.cpp"), (LAYER_BINDING, "layer_binding.cpp")):
        tmp = target + f".tmp{os.getpid()}"
        _compile(binding_command(source, tmp), tmp, target, verbose)
    with tempfile.TemporaryDirectory() as folder:
        objects = []
        for source in SOURCES + LAYER_SOURCES:
            objects.append(os.path.join(folder, source + ".o"))
            _compile(object_command(source, objects[-1]), objects[-1], objects[-1], verbose)
        tmp = LIB + f".tmp{os.getpid()}"
        _compile(link_command(objects, tmp), tmp, LIB, verbose)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
