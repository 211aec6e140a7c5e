"""Builds the CUDA library (sm_100a) in-tree with nvcc.  No JIT cache: the shared object sits
next to this file so that it travels with the source tree."""
from __future__ import annotations

import os
import shutil
import subprocess
import sys

PKG_DIR = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG_DIR)
CSRC = os.path.join(PKG_DIR, "csrc")
LIB_PATH = os.path.join(PKG_DIR, "libbetty.so")
SOURCES = ["api.cu", "vec.cu", "logreg.cu", "logreg_small.cu", "mlp.cu", "gemm.cu", "gemm_tc.cu", "block_norm.cu",
           "block_norm_bwd.cu", "act8.cu", "align.cu", "grouped.cu",
           "vocab_loss.cu", "vocab_products.cu"]
FAMILY_SOURCES = ["mlp.cu", "gemm.cu", "gemm_tc.cu"]
NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "--use_fast_math", "-Xcompiler", "-fPIC",
    "-I", os.path.join(ROOT, "include"), "-I", CSRC,
]


def _nvcc() -> str:
    for cand in (shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found: the CUDA library cannot be built")


def _stale() -> bool:
    if not os.path.exists(LIB_PATH):
        return True
    t = os.path.getmtime(LIB_PATH)
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC)] + [os.path.join(ROOT, "include", "betty.h"), __file__]
    return any(os.path.getmtime(d) > t for d in deps)


def _older(path: str, deps) -> bool:
    """Whether `path` is missing or older than any of `deps`."""
    return not os.path.exists(path) or any(os.path.getmtime(d) > os.path.getmtime(path) for d in deps)


def _unfinished(path: str) -> str:
    """Where the compiler writes: a file takes its place, and with it a date to be taken as fresh, only once it is whole."""
    return os.path.join(PKG_DIR, "_build", f"{os.path.basename(path)}.{os.getpid()}.part")


def _command(cmd, out: str):
    return subprocess.Popen(cmd + ["-o", _unfinished(out)], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)


def _finish(p, out: str):
    """Waits for the command; moves what it made into place.  Returns whether it succeeded, and its messages."""
    text, _ = p.communicate()
    if p.returncode == 0:
        os.replace(_unfinished(out), out)
    elif os.path.exists(_unfinished(out)):
        os.remove(_unfinished(out))
    return p.returncode == 0, text


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile every .cu of the package into libbetty.so; returns its path."""
    if not force and not _stale():
        return LIB_PATH
    nvcc = _nvcc()
    objs = []
    build_dir = os.path.join(PKG_DIR, "_build")
    os.makedirs(build_dir, exist_ok=True)
    procs = []
    headers = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".cuh")]
    headers += [os.path.join(ROOT, "include", "betty.h"), os.path.abspath(__file__)]
    # the MLP family sources are compiled twice: bfloat16 operands (default) and IEEE half operands
    units = [(src, "", []) for src in SOURCES] + [(src, "_f16", ["-DBETTY_FP16_OPERANDS"]) for src in FAMILY_SOURCES]
    for src, suffix, extra in units:
        obj = os.path.join(build_dir, src.replace(".cu", suffix + ".o"))
        objs.append(obj)
        if not force and not _older(obj, [os.path.join(CSRC, src)] + headers):
            continue
        cmd = [nvcc, "-c", os.path.join(CSRC, src)] + NVCC_FLAGS + extra
        if verbose:
            cmd += ["-Xptxas", "-v"]
        procs.append((src + suffix, obj, _command(cmd, obj)))
    failed = []
    for src, obj, p in procs:
        ok, out = _finish(p, obj)
        if not ok:
            failed.append(f"nvcc failed on {src}:\n{out}")
        elif verbose:
            print(out)
    if failed:
        raise RuntimeError("\n".join(failed))
    ok, out = _finish(_command([nvcc, "-shared"] + objs + ["-gencode", "arch=compute_100a,code=sm_100a"], LIB_PATH), LIB_PATH)
    if not ok:
        raise RuntimeError(f"link failed:\n{out}")
    return LIB_PATH


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
