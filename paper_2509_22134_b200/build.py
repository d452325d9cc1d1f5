"""Builds libgto.so (the C-ABI CUDA library) in-tree with nvcc for sm_100a, and _gto_decode.so (the
argument checks of the decoding-step calls, a Python extension beside it) with the host compiler."""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
OBJ = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libgto.so")
EXT = os.path.join(HERE, "_gto_decode.so")
EXT_KEY = os.path.join(OBJ, "_gto_decode.key")  # what EXT was built for
SOURCES = ["gto_api.cu", "row_reduce.cu", "tree_build.cu", "tree_reward.cu", "surrogate_grad.cu",
           "build_tree_noalloc.cu", "token_loss.cu", "decode_api.cu", "kv_cache.cu", "tree_verify.cu",
           "tree_attention_simt.cu", "tree_attention_tc.cu"]
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-lineinfo", "-std=c++17",
              "-Xcompiler", "-fPIC", "-Xptxas", "-v"]


def _nvcc() -> str:
    cand = os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "bin", "nvcc")
    return cand if os.path.exists(cand) else "nvcc"


def _stale(out: str, deps: list[str]) -> bool:
    if not os.path.exists(out):
        return True
    t = os.path.getmtime(out)
    return any(os.path.getmtime(d) > t for d in deps)


def extension_key() -> str:
    """What the extension is compiled against: it is stale, and not loaded, under another Python or PyTorch."""
    import sysconfig
    import torch
    return f"{sysconfig.get_config_var('SOABI')} torch {torch.__version__}"


def _extension_stale(deps: list[str]) -> bool:
    try:
        with open(EXT_KEY) as f:
            key = f.read()
    except OSError:
        return True
    return key != extension_key() or _stale(EXT, deps)


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile every kernel for sm_100a and link libgto.so; returns its path."""
    os.makedirs(OBJ, exist_ok=True)
    headers = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".h", ".cuh"))]
    headers.append(os.path.join(HERE, "..", "include", "gto.h"))
    jobs = []
    for src in SOURCES:
        s = os.path.join(CSRC, src)
        o = os.path.join(OBJ, src.replace(".cu", ".o"))
        if force or _stale(o, [s] + headers):
            jobs.append((s, o))

    def compile_one(job):
        s, o = job
        r = subprocess.run([_nvcc(), *NVCC_FLAGS, "-c", s, "-o", o], capture_output=True, text=True)
        log = o.replace(".o", ".ptxas.txt")
        with open(log, "w") as f:
            f.write(r.stderr)
        if r.returncode != 0:
            raise RuntimeError(f"nvcc failed on {s}:\n{r.stderr}")
        if verbose:
            sys.stderr.write(r.stderr)

    with ThreadPoolExecutor(max_workers=max(1, min(len(jobs), os.cpu_count() or 1))) as ex:
        list(ex.map(compile_one, jobs))
    objs = [os.path.join(OBJ, s.replace(".cu", ".o")) for s in SOURCES]
    if force or jobs or _stale(LIB, objs):
        r = subprocess.run([_nvcc(), "-shared", "-Xlinker", "-soname=libgto.so", "-o", LIB, *objs, "-cudart", "static", "-ldl"],
                           capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"link failed:\n{r.stderr}")
    src = os.path.join(CSRC, "decode_binding.cpp")
    if force or _extension_stale([src, headers[-1]]):
        import sysconfig
        import torch
        inc = os.path.join(os.path.dirname(torch.__file__), "include")
        r = subprocess.run(["g++", "-O2", "-std=c++17", "-fPIC", "-shared", src, "-o", EXT, "-I", inc, "-I",
                            os.path.join(inc, "torch", "csrc", "api", "include"), "-I",
                            sysconfig.get_paths()["include"],
                            f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
                            f'-DGTO_BUILT_FOR="{extension_key()}"',
                            LIB, "-Wl,-rpath,$ORIGIN", "-L", os.path.join(os.path.dirname(inc), "lib"),
                            "-ltorch_python", "-ltorch_cpu", "-lc10"], capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"g++ failed on {src}:\n{r.stderr}")
        with open(EXT_KEY, "w") as f:
            f.write(extension_key())
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose=True))
