"""Build the CUDA library in-tree: csrc/*.cu -> libsbc_b200.so (sm_100a only)."""
import concurrent.futures
import glob
import os
import shutil
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libsbc_b200.so")
OBJ = os.path.join(HERE, "_build")
NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17", "-Xcompiler", "-fPIC",
    # IEEE division and square root, no flush-to-zero
    "-ftz=false", "-prec-div=true", "-prec-sqrt=true",
]
# The method's kernels take their arithmetic as written (they are checked bit for bit): no fused
# multiply-add contraction.  The language-model operators are held to tolerances and may fuse.
SOURCES = {"sbc_api.cu": ["-fmad=false"], "lm_api.cu": []}


def _nvcc() -> str:
    path = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(path):
        raise RuntimeError("nvcc not found: the CUDA library cannot be built")
    return path


def needs_build() -> bool:
    if not os.path.exists(LIB):
        return True
    deps = glob.glob(os.path.join(CSRC, "*")) + glob.glob(os.path.join(HERE, "..", "include", "*.h"))
    return any(os.path.getmtime(d) > os.path.getmtime(LIB) for d in deps)


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and not needs_build():
        return LIB
    os.makedirs(OBJ, exist_ok=True)
    extra = ["-Xptxas", "-v"] if verbose else []

    def compile_one(item):
        source, flags = item
        obj = os.path.join(OBJ, source.replace(".cu", ".o"))
        subprocess.run([_nvcc(), *NVCC_FLAGS, *flags, *extra, "-c", "-o", obj, os.path.join(CSRC, source)], check=True, cwd=CSRC)
        return obj

    with concurrent.futures.ThreadPoolExecutor(len(SOURCES)) as pool:
        objects = list(pool.map(compile_one, SOURCES.items()))
    subprocess.run([_nvcc(), *NVCC_FLAGS, "-shared", "-o", LIB, *objects], check=True, cwd=CSRC)
    return LIB


if __name__ == "__main__":
    print(build(force=True, verbose=True))
