"""Compile the CUDA library in-tree for sm_100a with nvcc (works without a GPU), and the native marshalling of torch tensors with g++."""
from __future__ import annotations

import os
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor
from pathlib import Path

HERE = Path(__file__).resolve().parent
CSRC = HERE / "csrc"
INCLUDE = HERE.parent / "include"
LIB = HERE / "libpsa.so"
CALLS = HERE / "_torch_calls.so"      # a Python extension module (csrc/torch_calls.cpp)
SOURCES = ["api.cu", "plan.cpp", "prefix_sm100.cu", "suffix_sm100.cu", "merge_sm100.cu", "static_workspace.cu", "append_sm100.cu", "sample_sm100.cu", "attn_tasks.cu",
           "pages_sm100.cu", "kv4_sm100.cu", "suffix_kv4_sm100.cu", "logits_sm100.cu", "chunk_sm100.cu", "store_sm100.cu", "weights_sm100.cu", "evict_sm100.cu",
           "logprobs_sm100.cu"]
NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "-Xcompiler", "-fPIC", "-Xptxas", "-v", f"-I{INCLUDE}", f"-I{CSRC}",
]


def _nvcc() -> str:
    cand = os.environ.get("NVCC") or "/usr/local/cuda/bin/nvcc"
    return cand if Path(cand).exists() else "nvcc"


def _stale(target: Path, deps) -> bool:
    if not target.exists():
        return True
    t = target.stat().st_mtime
    return any(Path(d).stat().st_mtime > t for d in deps)


def build(force: bool = False, verbose: bool = False) -> Path:
    headers = list(CSRC.glob("*.h")) + list(CSRC.glob("*.cuh")) + list(INCLUDE.glob("*.h"))
    objdir = HERE / "_build"
    objdir.mkdir(exist_ok=True)
    logs = {}

    def compile_one(src: str):
        obj = objdir / (src.rsplit(".", 1)[0] + ".o")
        if force or _stale(obj, [CSRC / src, *headers]):
            cmd = [_nvcc(), *NVCC_FLAGS, "-x", "cu", "-c", str(CSRC / src), "-o", str(obj)]
            r = subprocess.run(cmd, capture_output=True, text=True)
            logs[src] = r.stderr + r.stdout
            if r.returncode != 0:
                raise RuntimeError(f"nvcc failed on {src}:\n{logs[src]}")
        return obj

    def compile_calls():
        src = CSRC / "torch_calls.cpp"
        if not (force or _stale(CALLS, [src, *INCLUDE.glob("*.h")])):
            return
        import torch
        torch_dir = Path(torch.__file__).resolve().parent
        tmp = CALLS.with_suffix(f".tmp{os.getpid()}.so")
        cuda = Path(_nvcc()).resolve().parent.parent / "include"
        cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", f"-I{INCLUDE}",
               "-isystem", str(torch_dir / "include"), "-isystem", str(torch_dir / "include/torch/csrc/api/include"),
               "-isystem", sysconfig.get_path("include"), "-isystem", str(cuda), str(src), "-o", str(tmp),
               f"-L{torch_dir / 'lib'}", "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_cuda", "-ldl"]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"g++ failed on {src.name}:\n{r.stderr}")
        os.replace(tmp, CALLS)

    with ThreadPoolExecutor(max_workers=len(SOURCES) + 1) as ex:
        calls = ex.submit(compile_calls)
        objs = list(ex.map(compile_one, SOURCES))
        calls.result()
    if force or _stale(LIB, objs):
        tmp = LIB.with_suffix(f".tmp{os.getpid()}.so")
        cmd = [_nvcc(), "-shared", "-gencode", "arch=compute_100a,code=sm_100a", "-o", str(tmp), *map(str, objs), "-ldl"]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"link failed:\n{r.stderr}")
        os.replace(tmp, LIB)
    if verbose:
        for src, log in logs.items():
            print(f"==== {src}\n{log}")
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose=True))
