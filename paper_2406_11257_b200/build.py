"""Builds the CUDA library in-tree: csrc/*.cu -> libexcp.so (sm_100a only), and the native half of the Python
binding of the scoring calls: csrc/score_binding.cpp -> _score-<hash>.so (against the installed torch)."""
from __future__ import annotations

import hashlib
import os
import shutil
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libexcp.so")
SOURCES = ["stats.cu", "mask_compact.cu", "kmeans.cu", "pack.cu", "decode.cu", "excp_api.cu", "excp_noalloc.cu", "selftest.cu",
           "mx4.cu", "mx4_matmul.cu", "mx4_matmul_wide.cu", "token_logprobs.cu", "score_api.cu",
           "act8.cu", "layer_norm.cu", "product.cu", "product_wide.cu", "layers_api.cu"]
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-fmad=false", "-Xcompiler", "-fPIC", "-cudart", "static"]


def extra_flags() -> list[str]:
    """Extra nvcc flags from the environment (EXCP_NVCC_FLAGS), e.g. -DEXCP_DEBUG_BOUNDS for the build in which what
    compresses and restores checks every index it forms and reports through the call's status instead of faulting."""
    return os.environ.get("EXCP_NVCC_FLAGS", "").split()


def lib_path() -> str:
    """libexcp.so for the plain build; a build with extra flags gets a name of its own (and its own objects), so
    that it never replaces the plain library."""
    flags = extra_flags()
    if not flags:
        return LIB
    return os.path.join(HERE, "libexcp-" + hashlib.sha1(" ".join(flags).encode()).hexdigest()[:8] + ".so")


def _stale(lib: str) -> bool:
    if not os.path.exists(lib):
        return True
    t = os.path.getmtime(lib)
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".cu", ".cuh", ".h"))]
    deps.append(os.path.join(os.path.dirname(HERE), "include", "excp.h"))
    return any(os.path.getmtime(d) > t for d in deps)


def binding_path() -> str:
    """The native half of the scoring calls' binding.  Its name carries what it is compiled against: under another Python
    or torch it is another file, and neither takes the other's."""
    import torch
    key = f"{sysconfig.get_config_var('SOABI')} {torch.__version__} {int(torch._C._GLIBCXX_USE_CXX11_ABI)}"
    return os.path.join(HERE, "_score-" + hashlib.sha1(key.encode()).hexdigest()[:8] + ".so")


def build_binding(force: bool = False) -> str:
    """Compiles binding_path() if it is missing or older than its sources; returns it."""
    import torch
    out = binding_path()
    deps = [os.path.join(CSRC, "score_binding.cpp"), os.path.join(os.path.dirname(HERE), "include", "excp.h")]
    if not force and os.path.exists(out) and all(os.path.getmtime(d) <= os.path.getmtime(out) for d in deps):
        return out
    at = os.path.dirname(torch.__file__)
    nvcc = os.environ.get("NVCC", "nvcc")
    cuda = os.path.dirname(os.path.dirname(os.path.realpath(shutil.which(nvcc) or "/usr/local/cuda/bin/nvcc")))
    include = [os.path.join(at, "include"), sysconfig.get_paths()["include"], os.path.join(cuda, "include")]
    part = out + f".{os.getpid()}"
    subprocess.check_call([os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared",
                           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", *["-I" + i for i in include], deps[0], "-o", part,
                           "-L" + os.path.join(at, "lib"), "-ltorch_python", "-ltorch", "-ltorch_cpu", "-lc10", "-lc10_cuda", "-ltorch_cuda"])
    os.replace(part, out)      # whole or not at all: another process may be loading it
    return out


def build(force: bool = False, verbose: bool = False) -> str:
    """Compiles the library if it is missing or older than its sources; returns its path."""
    lib = lib_path()
    if not force and not _stale(lib):
        return lib
    tag = os.path.basename(lib)[len("libexcp"):-len(".so")]        # "" or "-<hash>"
    nvcc = os.environ.get("NVCC", "nvcc")
    objs = []
    procs = []
    for src in SOURCES:
        obj = os.path.join(CSRC, src[:-3] + tag + ".o")
        cmd = [nvcc, *NVCC_FLAGS, *extra_flags(), "-c", os.path.join(CSRC, src), "-o", obj]
        if verbose:
            cmd.insert(1, "-Xptxas=-v")
        procs.append((src, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
        objs.append(obj)
    failed = False
    for src, p in procs:
        out, _ = p.communicate()
        if p.returncode != 0 or verbose:
            sys.stderr.write(f"--- {src}\n{out}\n")
        failed |= p.returncode != 0
    if failed:
        raise RuntimeError("nvcc failed")
    subprocess.check_call([nvcc, "-shared", "-gencode", "arch=compute_100a,code=sm_100a", "-cudart", "static", "-o", lib, *objs, "-lrt", "-ldl", "-lpthread"])
    return lib


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
    print(build_binding(force="--force" in sys.argv))
