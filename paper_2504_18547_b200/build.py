"""Builds libvitint.so (sm_100a) in-tree with nvcc.  No GPU is needed to compile."""
from __future__ import annotations

import subprocess
from pathlib import Path

PKG = Path(__file__).resolve().parent
CSRC = PKG / "csrc"
LIB = PKG / "libvitint.so"
INCLUDE = PKG.parent / "include"

NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17", "-Xcompiler", "-fPIC"]

# The library's translation units; each includes the .cu files of its part (see the files).
UNITS = {"vitint_lib": ["api", "params", "quantize", "layernorm_compare", "softmax", "gemm", "gemm_direct", "attention_fused", "attention_long",
                        "attention", "softmax_table", "encoder", "selftest", "linear_e2m1"],
         "cache_lib": ["qk_norm_rotate", "cache_evict", "paged_attention", "paged_attention_tiles", "cache_weigh"]}


def sources():
    return sorted(CSRC.glob("*.cu")) + sorted(CSRC.glob("*.cuh")) + [INCLUDE / "vitint.h"]


def unit_sources(unit: str):
    """What a translation unit is compiled from: its .cu files and every header."""
    return [CSRC / f"{name}.cu" for name in [unit, *UNITS[unit]]] + sorted(CSRC.glob("*.cuh")) + [INCLUDE / "vitint.h"]


def needs_build() -> bool:
    if not LIB.exists():
        return True
    t = LIB.stat().st_mtime
    return any(p.stat().st_mtime > t for p in sources())


def _compile_and_link(out: Path, tag: str, flags, force: bool) -> None:
    """Compiles the units side by side (an object newer than its sources stays) and links them."""
    objects, running = [], []
    for unit in UNITS:
        obj = CSRC / f"{unit}{tag}.o"
        objects.append(obj)
        if force or not obj.exists() or any(p.stat().st_mtime > obj.stat().st_mtime for p in unit_sources(unit)):
            cmd = ["nvcc", *NVCC_FLAGS, *flags, f"-I{INCLUDE}", "-c", str(CSRC / f"{unit}.cu"), "-o", str(obj)]
            running.append((obj, cmd, subprocess.Popen(cmd)))
    failed = [(obj, cmd, rc) for obj, cmd, rc in [(obj, cmd, p.wait()) for obj, cmd, p in running] if rc != 0]
    for obj, _, _ in failed:
        obj.unlink(missing_ok=True)
    if failed:
        raise subprocess.CalledProcessError(failed[0][2], failed[0][1])
    subprocess.run(["nvcc", *NVCC_FLAGS[:2], "-shared", *map(str, objects), "-o", str(out)], check=True)


def build_library(force: bool = False, verbose: bool = False) -> Path:
    if force or needs_build():
        _compile_and_link(LIB, "", ["-Xptxas=-v"] if verbose else [], force)
    return LIB


TRACE_LIB = PKG / "libvitint_trace.so"


def build_trace_library() -> Path:
    """Diagnostic build (-DVITINT_TRACE): the GEMM kernel records a timeline of its warp roles (see trace_gemm.py).
    A separate file; the product library is never built with the flag."""
    _compile_and_link(TRACE_LIB, "_trace", ["-DVITINT_TRACE"], True)
    return TRACE_LIB


if __name__ == "__main__":
    print(build_library(force=True, verbose=True))
