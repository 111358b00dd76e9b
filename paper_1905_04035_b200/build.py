"""Build the CUDA library in-tree with nvcc for sm_100a (no JIT cache, no pip install)."""
from __future__ import annotations

import os
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIB_PATH = os.path.join(HERE, "libdst_b200.so")
CALLS_SOURCE = os.path.join(CSRC, "dst_python.cpp")  # the entries as a Python module (binding.calls_path())
SOURCES = ["dst_api.cu", "dst_index_kernels.cu", "dst_front_cluster.cu", "dst_reduce_kernels.cu",
           "dst_accumulate_kernels.cu", "dst_dropout.cu", "dst_fp8.cu", "dst_fp4.cu", "dst_sample.cu", "dst_tied_api.cu",
           "dst_logprob.cu", "dst_norm.cu", "dst_clip.cu", "dst_step_api.cu"]
HEADERS = [os.path.join(CSRC, h) for h in ("dst_common.cuh", "dst_tied.cuh", "dst_async.cuh", "dst_fp8.cuh", "dst_fp4.cuh", "dst_block_matmul.cuh", "dst_step.cuh")] + [
    os.path.join(INCLUDE, h) for h in ("dst.h", "dst_tied.h", "dst_step.h")]
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xcompiler", "-fPIC", "-I", INCLUDE]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if cand and (os.path.sep not in cand or os.path.exists(cand)):
            return cand
    return "nvcc"


def _older(path: str, deps) -> bool:
    return not os.path.exists(path) or any(os.path.getmtime(p) > os.path.getmtime(path) for p in deps)


def stale_parts():
    """Whether the library, and the Python module of its entries, are to be built: missing, older than their sources, or such as do not load."""
    from . import binding
    library = _older(LIB_PATH, [os.path.join(CSRC, s) for s in SOURCES] + HEADERS)
    calls = library or _older(binding.calls_path(), [CALLS_SOURCE] + HEADERS)
    if not library:                                   # (what is to be built anew is not loaded before)
        try:
            binding.load_library()
            if not calls:
                binding.load_calls()
        except ImportError:
            calls = True
        except (OSError, AttributeError):
            library = calls = True
    return library, calls


def is_stale() -> bool:
    return any(stale_parts())


def _calls_commands(obj: str, out: str):
    """The compiler's command for the Python module, and the linker's."""
    import torch

    base = os.path.join(os.path.dirname(torch.__file__), "include")
    include = [INCLUDE, sysconfig.get_paths()["include"], base, os.path.join(base, "torch", "csrc", "api", "include")]
    flags = ["-O2", "-std=c++17", "-fPIC", "-fvisibility=hidden", "-D_GLIBCXX_USE_CXX11_ABI=%d" % torch.compiled_with_cxx11_abi()]
    libs = os.path.join(os.path.dirname(torch.__file__), "lib")
    return (["g++"] + flags + [a for i in include for a in ("-I", i)] + ["-c", CALLS_SOURCE, "-o", obj],
            ["g++", "-shared", "-o", out, obj, "-L" + HERE, "-l:" + os.path.basename(LIB_PATH), "-Wl,-rpath,$ORIGIN", "-L" + libs, "-ltorch_python", "-ltorch_cpu", "-lc10"])


def build_library(force: bool = False, verbose: bool = False) -> str:
    """Compile every .cu file and link ``libdst_b200.so`` next to this file, and the Python module of its entries; of the two, what is stale."""
    from . import binding
    library, calls = (True, True) if force else stale_parts()
    objdir = os.path.join(HERE, "_build")
    os.makedirs(objdir, exist_ok=True)
    nvcc = _nvcc()
    procs = []
    objs = []
    for s in SOURCES if library else []:
        obj = os.path.join(objdir, s[:-3] + ".o")
        cmd = [nvcc] + NVCC_FLAGS + (["-Xptxas", "-v"] if verbose else []) + ["-c", os.path.join(CSRC, s), "-o", obj]
        procs.append((cmd, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
        objs.append(obj)
    tag = ".tmp.%d" % os.getpid()
    calls_path = binding.calls_path()
    compile_calls, link_calls = _calls_commands(os.path.join(objdir, "dst_python.o"), calls_path + tag)
    if calls:
        procs.append((compile_calls, subprocess.Popen(compile_calls, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    for cmd, p in procs:
        out, _ = p.communicate()
        if verbose or p.returncode != 0:
            sys.stderr.write(out)
        if p.returncode != 0:
            raise RuntimeError("compilation failed: %s" % " ".join(cmd))
    if library:
        tmp = LIB_PATH + tag
        subprocess.check_call([nvcc, "-shared", "-o", tmp] + objs + ["-gencode", "arch=compute_100a,code=sm_100a", "-ldl"])
        os.replace(tmp, LIB_PATH)
    if calls:
        subprocess.check_call(link_calls)
        os.replace(calls_path + tag, calls_path)
    return LIB_PATH


if __name__ == "__main__":
    print(build_library(force="--force" in sys.argv, verbose="-v" in sys.argv))
