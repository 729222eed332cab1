"""Build libjakiro.so (nvcc, sm_100a, cross-compiles without a GPU) and _calls.so (g++, against torch) in-tree."""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(os.path.dirname(HERE), "include")
LIB = os.path.join(HERE, "libjakiro.so")
CALLS = os.path.join(HERE, "_calls.so")
BUILD_DIR = os.path.join(HERE, "_build")
CALLS_FOR = os.path.join(BUILD_DIR, "calls_built_for")     # the versions that _calls.so was built for
SOURCES = ["jk_api.cu", "jk_expand.cu", "jk_gemm_tc.cu", "jk_attn.cu", "jk_attn_tc.cu", "jk_attn_sk.cu", "jk_attn_cl.cu",
           "jk_accept.cu", "jk_pre.cu", "jk_paged.cu", "jk_paged_attn.cu", "jk_paged_tc.cu", "jk_sample.cu",
           "jk_norm.cu", "jk_rope.cu", "jk_linear.cu", "jk_linear_tc.cu", "jk_linear_pair.cu"]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if cand and (os.path.isabs(cand) and os.path.exists(cand) or not os.path.isabs(cand)):
            return cand
    raise RuntimeError("nvcc not found")


def _older(target: str, sources) -> bool:
    """Is the target missing, or older than one of its sources?"""
    return not os.path.exists(target) or any(os.path.getmtime(d) > os.path.getmtime(target) for d in sources)


def _built_for() -> str:
    """What _calls.so holds for: it is tied to one Python and one torch, the library to neither."""
    import torch
    return f"{sys.implementation.cache_tag} {torch.__version__} {int(torch._C._GLIBCXX_USE_CXX11_ABI)}\n"


def library_needs_build() -> bool:
    return _older(LIB, [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f != "jk_calls.cpp"] + [os.path.join(INCLUDE, "jakiro.h")])


def calls_need_build() -> bool:
    if _older(CALLS, [os.path.join(CSRC, "jk_calls.cpp"), os.path.join(INCLUDE, "jakiro.h")]) or not os.path.exists(CALLS_FOR):
        return True
    with open(CALLS_FOR) as f:
        return f.read() != _built_for()


def needs_build() -> bool:
    return library_needs_build() or calls_need_build()


def _calls_command() -> list:
    import sysconfig

    import torch
    from torch.utils import cpp_extension
    cuda = os.path.dirname(os.path.dirname(_nvcc()))
    dirs = cpp_extension.include_paths() + [sysconfig.get_paths()["include"], os.path.join(cuda, "include"), INCLUDE]
    libs = os.path.join(os.path.dirname(torch.__file__), "lib")
    return (["g++", "-std=c++17", "-O2", "-fPIC", "-shared", "-w", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}"]
            + [f"-I{d}" for d in dirs] + [os.path.join(CSRC, "jk_calls.cpp"), "-o", CALLS, f"-L{libs}"]
            + [f"-l{n}" for n in ("torch_python", "torch_cpu", "c10", "c10_cuda")])


def _finish(name: str, p: subprocess.Popen, verbose: bool) -> None:
    out, _ = p.communicate()
    if verbose or p.returncode:
        sys.stderr.write(out.decode())
    if p.returncode:
        raise RuntimeError(f"the compiler failed on {name}")


def build(force: bool = False, verbose: bool = False) -> str:
    """Builds what is missing, older than its sources or, of _calls.so, made for another Python or torch.  The library is
    there, and all calls but the target layer's work from Python, even where _calls.so cannot be built."""
    library, calls = force or library_needs_build(), force or calls_need_build()
    os.makedirs(BUILD_DIR, exist_ok=True)
    pipes = dict(stdout=subprocess.PIPE, stderr=subprocess.STDOUT)
    procs = []
    if library:
        common = [_nvcc(), "-std=c++17", "-O3", "-lineinfo", "-gencode",
                  "arch=compute_100a,code=sm_100a", "-Xcompiler", "-fPIC", "-I", INCLUDE, "-I", CSRC]
        if verbose:
            common += ["-Xptxas", "-v"]
        objs = [os.path.join(BUILD_DIR, src.replace(".cu", ".o")) for src in SOURCES]
        procs = [(src, subprocess.Popen(common + ["-c", os.path.join(CSRC, src), "-o", obj], **pipes))
                 for src, obj in zip(SOURCES, objs)]
    extension = subprocess.Popen(_calls_command(), **pipes) if calls else None
    for src, p in procs:
        _finish(src, p, verbose)
    if library:
        subprocess.check_call([_nvcc(), "-shared", "-o", LIB] + objs + ["-cudart", "static"])
    if calls:
        _finish("jk_calls.cpp", extension, verbose)
        with open(CALLS_FOR, "w") as f:
            f.write(_built_for())
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
