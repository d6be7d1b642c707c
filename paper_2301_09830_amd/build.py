"""Build liboptcc.so (HIP, gfx950) in-tree with hipcc.

    python -m paper_2301_09830_amd.build        # or build() from Python

The library has two translation units: csrc/api.hip (the compressor) and
csrc/stage_ops.hip (the operators a pipeline stage runs beside it), compiled
side by side and linked.  Packed-fp32 VALU instructions are disabled for the
device code.  The binding of the layers, csrc/bind_layers.cpp, is host code
against torch's headers: a Python module beside the library.
"""

from __future__ import annotations

import os
import shutil
import subprocess
import sys
import sysconfig

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIB = os.path.join(PKG, "liboptcc.so")
LAYERS = os.path.join(PKG, "_layers.so")
ARCH = "gfx950"


def hipcc() -> str:
    for cand in (shutil.which("hipcc"), "/opt/rocm/bin/hipcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("hipcc not found (ROCm is required to build liboptcc)")


SOURCES = ("api.hip", "stage_ops.hip")


def compile_command(out: str = LIB, source: str = SOURCES[0]) -> list:
    """hipcc's command for one translation unit, as a shared library."""
    return [
        hipcc(), f"--offload-arch={ARCH}", "-O3", "-std=c++17", "-fPIC", "-shared",
        "-ffp-contract=off",
        "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
        "-Wno-unused-result",
        "-I", INCLUDE, "-I", CSRC,
        os.path.join(CSRC, source),
        "-o", out,
    ]


def layers_command(out: str = LAYERS) -> list:
    """g++'s command for the binding of the layers."""
    import torch
    home = os.path.dirname(torch.__file__)
    include = os.path.join(home, "include")
    return [
        "g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden",
        f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
        "-I", INCLUDE, "-isystem", include,
        "-isystem", os.path.join(include, "torch", "csrc", "api", "include"),
        "-isystem", sysconfig.get_paths()["include"],
        os.path.join(CSRC, "bind_layers.cpp"),
        "-L", os.path.join(home, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10",
        "-o", out,
    ]


def build(verbose: bool = False) -> str:
    """Compile liboptcc.so for gfx950 and, where torch is installed, the binding
    of the layers next to this file; returns the library's path."""
    tmp = LIB + ".tmp"
    objects = [LIB + f".{i}.o" for i in range(len(SOURCES))]
    steps = [[c for c in compile_command(o, src) if c != "-shared"] + ["-c"]
             for o, src in zip(objects, SOURCES)]
    try:
        steps.append(layers_command(LAYERS + ".tmp"))
    except ImportError:   # no torch: the library alone, for programs of its C interface
        pass
    try:
        procs = [subprocess.Popen(cmd, stdout=subprocess.DEVNULL, stderr=subprocess.PIPE, text=True)
                 for cmd in steps]
        for proc, cmd, err in [(p, c, p.communicate()[1]) for p, c in zip(procs, steps)]:
            _report(proc.returncode, cmd, err, verbose)
        link = [hipcc(), f"--offload-arch={ARCH}", "-fPIC", "-shared", *objects, "-o", tmp]
        proc = subprocess.run(link, capture_output=True, text=True)
        _report(proc.returncode, link, proc.stderr, verbose)
    finally:
        for o in objects:
            if os.path.exists(o):
                os.remove(o)
    if len(steps) > len(SOURCES):
        os.replace(LAYERS + ".tmp", LAYERS)
    os.replace(tmp, LIB)
    return LIB


def _report(code: int, cmd: list, err: str, verbose: bool) -> None:
    noise = "is not a recognized feature for this target"
    lines = [ln for ln in err.splitlines() if noise not in ln]
    if code != 0:
        raise RuntimeError("compiler failed:\n" + " ".join(cmd) + "\n" + "\n".join(lines))
    if verbose and lines:
        print("\n".join(lines), file=sys.stderr)


if __name__ == "__main__":
    print(build(verbose=True))
