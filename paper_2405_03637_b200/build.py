"""Builds the CUDA library in-tree with nvcc for sm_100a (cross-compiles without a GPU).

    python -m paper_2405_03637_b200.build [--force] [--verbose] [--define NAME[=VALUE]]... [--out PATH]

--define adds a preprocessor definition (the geometry constants COLLAGE_PIPE_* / COLLAGE_FP32_*, or
COLLAGE_DATA_MOVEMENT_ONLY, which compiles the arithmetic out of the step kernel to measure what the
copy pipeline alone sustains); such a build goes to --out, never over the in-tree library, and is
loaded only on request: `binding.load(path)`, which `bench.py --lib PATH` calls.

The exactness of the error-free transforms depends on the flags below: no FMA contraction,
no flush-to-zero, IEEE division and square root, never --use_fast_math.
"""
from __future__ import annotations

import os
import subprocess
import sys
from pathlib import Path

HERE = Path(__file__).resolve().parent
CSRC = HERE / "csrc"
LIB = HERE / "libcollage_b200.so"
SOURCES = ["collage_step.cu", "collage_primitives.cu", "collage_edq_static.cu", "collage_fp32_master.cu"]
# The training-step operators, each file compiled in one piece and the files at once.  (Split compilation, as below, gave one
# of two codes from the same file, from build to build: up to a tenth of a kernel's time.)
OPERATOR_SOURCES = ["row_norm.cu", "gated_ffn.cu", "distill_loss.cu", "block_norm.cu", "token_loss.cu", "adam_multi.cu"]
NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "-fmad=false", "-ftz=false", "-prec-div=true", "-prec-sqrt=true",
    "-Xcompiler", "-fPIC", "-cudart", "static",
]
SPLIT_FLAGS = ["--split-compile", "0", "-t", "0"]      # compile the many kernel instantiations on all host cores


def _newest_source_mtime() -> float:
    files = list(CSRC.glob("*.cu")) + list(CSRC.glob("*.cuh")) + [HERE.parent / "include" / "collage.h", Path(__file__)]
    return max(f.stat().st_mtime for f in files)


def build(force: bool = False, verbose: bool = False, defines: tuple = (), out: Path | None = None) -> Path:
    if defines and out is None:
        raise ValueError("a build with extra definitions needs its own output path")
    lib = Path(out) if out is not None else LIB
    if out is None and not force and LIB.exists() and LIB.stat().st_mtime >= _newest_source_mtime():
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    tmp = lib.with_suffix(f".so.tmp{os.getpid()}")
    extra = [*[f"-D{d}" for d in defines], *(["-Xptxas", "-v"] if verbose else [])]
    objects = [lib.parent / f"{Path(s).stem}.tmp{os.getpid()}.o" for s in OPERATOR_SOURCES]
    try:
        procs = [subprocess.Popen([nvcc, *NVCC_FLAGS, *extra, "-c", "-o", str(o), str(CSRC / s)], stdout=subprocess.PIPE,
                                  stderr=subprocess.STDOUT, text=True) for s, o in zip(OPERATOR_SOURCES, objects)]
        done = [(p.communicate()[0], p.returncode) for p in procs]
        if all(rc == 0 for _, rc in done):
            p = subprocess.run([nvcc, *NVCC_FLAGS, *SPLIT_FLAGS, *extra, "-shared", "-o", str(tmp), *[str(CSRC / s) for s in SOURCES],
                                *[str(o) for o in objects]], capture_output=True, text=True)
            done.append((p.stdout + p.stderr, p.returncode))
    finally:
        for o in objects:
            o.unlink(missing_ok=True)
    failed = any(rc for _, rc in done)
    if verbose or failed:
        sys.stderr.write("".join(text for text, _ in done))
    if failed:
        raise RuntimeError("nvcc failed building the Collage CUDA library")
    os.replace(tmp, lib)
    return lib


if __name__ == "__main__":
    argv = sys.argv[1:]
    defs = tuple(argv[i + 1] for i, a in enumerate(argv) if a == "--define" and i + 1 < len(argv))
    outp = next((Path(argv[i + 1]) for i, a in enumerate(argv) if a == "--out" and i + 1 < len(argv)), None)
    print(build(force="--force" in argv, verbose="--verbose" in argv, defines=defs, out=outp))
