"""Build the CUDA library libmpadam.so for sm_103a (GB300), in tree, and the
Python module _mpadam_torch beside it (tensor marshalling in C++, for the
installed torch).

Each translation unit compiles in its own compiler process (in parallel), then
one call links each of the two.  Output: paper_2607_10611_gb300/_build/.
"""
from __future__ import annotations

import importlib.machinery
import importlib.metadata
import importlib.util
import os
import shutil
import subprocess
import sysconfig
from concurrent.futures import ThreadPoolExecutor
from pathlib import Path

PKG = Path(__file__).resolve().parent
ROOT = PKG.parent
CSRC = PKG / "csrc"
INCLUDE = ROOT / "include"
OUT_DIR = PKG / "_build"
LIB = OUT_DIR / "libmpadam.so"
EXT = OUT_DIR / "_mpadam_torch.so"
EXT_SOURCE = "torch_ext.cpp"
EXT_TORCH = OUT_DIR / "torch_version"  # the torch that EXT was built for

SOURCES = ["mpadam_api.cu", "step_bf16.cu", "step_e4m3.cu", "step_e4m3b.cu", "step_nvfp4.cu", "toy.cu",
           "train_api.cu", "adamw.cu", "fp8_quant.cu", "fp8_matmul.cu"]
HEADERS = ["step_args.h", "step_kernel.cuh", "toy.h", "host.h", "adamw.h", "adamw_math.cuh", "fp8.h", "launch.h"]

ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
NVCC_FLAGS = ARCH + [
    "-O3", "-lineinfo", "-std=c++17", "-Xcompiler", "-fPIC",
    # every float op in the kernels is an explicit _rn intrinsic; these keep
    # any other floating-point code IEEE as well
    "-fmad=false", "--ftz=false", "--prec-div=true", "--prec-sqrt=true",
    "-DNDEBUG", f"-I{INCLUDE}", f"-I{CSRC}",
]


def nvcc() -> str:
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and Path(cand).exists():
            return cand
    raise RuntimeError("nvcc not found")


def _inputs():
    return [CSRC / s for s in SOURCES + [EXT_SOURCE]] + [CSRC / h for h in HEADERS] + [INCLUDE / "mpadam.h", Path(__file__)]


def needs_build() -> bool:
    if not LIB.exists() or not EXT.exists() or not EXT_TORCH.exists():
        return True
    if EXT_TORCH.read_text() != importlib.metadata.version("torch"):
        return True
    t = LIB.stat().st_mtime
    return any(p.stat().st_mtime > t for p in _inputs())


def _torch_dir() -> Path:
    return Path(importlib.util.find_spec("torch").origin).parent


def _ext_flags():
    inc = _torch_dir() / "include"
    cuda = Path(nvcc()).resolve().parent.parent / "include"
    return ["-O2", "-std=c++17", "-fPIC", "-DNDEBUG", f"-I{INCLUDE}", f"-I{inc}",
            f"-I{inc / 'torch' / 'csrc' / 'api' / 'include'}", f"-I{sysconfig.get_paths()['include']}", f"-I{cuda}"]


def build(force: bool = False, verbose: bool = False, ptxas_info: bool = False) -> Path:
    if not force and not needs_build():
        return LIB
    OUT_DIR.mkdir(exist_ok=True)
    cc = nvcc()
    extra = ["-Xptxas", "-v"] if ptxas_info else []

    def compile_one(src: str):
        obj = OUT_DIR / (Path(src).stem + ".o")
        cmd = [cc, *NVCC_FLAGS, *extra, "-c", str(CSRC / src), "-o", str(obj)]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"nvcc failed for {src}:\n{r.stdout}\n{r.stderr}")
        return obj, r.stdout + r.stderr

    def compile_ext():
        obj = OUT_DIR / (Path(EXT_SOURCE).stem + ".o")
        cmd = [os.environ.get("CXX", "g++"), *_ext_flags(), "-c", str(CSRC / EXT_SOURCE), "-o", str(obj)]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"compilation failed for {EXT_SOURCE}:\n{r.stdout}\n{r.stderr}")
        return obj

    with ThreadPoolExecutor(max_workers=len(SOURCES) + 1) as ex:
        ext = ex.submit(compile_ext)
        results = list(ex.map(compile_one, SOURCES))
        ext_obj = ext.result()
    if verbose or ptxas_info:
        for _, log in results:
            if log.strip():
                print(log)
    tmp = OUT_DIR / f".libmpadam.{os.getpid()}.so"
    cmd = [cc, *ARCH, "-shared", "-o", str(tmp), *[str(o) for o, _ in results]]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stdout}\n{r.stderr}")
    EXT_TORCH.unlink(missing_ok=True)  # until EXT is linked against this LIB, the build is not done
    os.replace(tmp, LIB)
    tmp = OUT_DIR / f".mpadam_torch.{os.getpid()}.so"
    cmd = [os.environ.get("CXX", "g++"), "-shared", "-o", str(tmp), str(ext_obj), f"-L{_torch_dir() / 'lib'}",
           "-ltorch_python", "-ltorch_cpu", "-lc10_cuda", "-lc10", f"-L{OUT_DIR}", "-l:libmpadam.so",
           "-Wl,-rpath,$ORIGIN"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link of {EXT.name} failed:\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, EXT)
    EXT_TORCH.write_text(importlib.metadata.version("torch"))
    return LIB


def load_ext():
    """The module _mpadam_torch; there is no fallback."""
    import torch  # noqa: F401  (its libraries have to be loaded first)
    if not EXT.exists():
        raise RuntimeError(f"{EXT} is missing: build the CUDA library first (paper_2607_10611_gb300.build())")
    spec = importlib.util.spec_from_loader("_mpadam_torch", importlib.machinery.ExtensionFileLoader("_mpadam_torch", str(EXT)))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


if __name__ == "__main__":
    import sys
    print(build(force=True, ptxas_info="-v" in sys.argv))
