"""Build the in-tree shared library libsn.so (C ABI + sm_103a kernels).

Every translation unit under csrc/ is compiled by nvcc in parallel for
sm_103a only, then linked with the static CUDA runtime into libsn.so next to
this file.  Host code is portable C++17 (x86_64 here, aarch64 on the GPU host).
bind/*.cpp, the tensor front end of the block and attention operators, is compiled
beside them against PyTorch's headers and linked to libsn.so as the module _blocks,
where PyTorch is installed: the library itself needs nvcc alone.
"""
from __future__ import annotations

import concurrent.futures as cf
import glob
import importlib.util
import os
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
BUILD = os.path.join(CSRC, "_build")
LIB = os.path.join(HERE, "libsn.so")
BIND_DIR = os.path.join(HERE, "bind")
BIND = os.path.join(HERE, "_blocks.so")
NVCC = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
FLAGS = ["-O3", "-std=c++17", "-lineinfo", "-Xcompiler", "-fPIC", "-Xcompiler", "-fvisibility=hidden",
         "--expt-relaxed-constexpr", "-I", os.path.join(HERE, "..", "include")]


def _sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")) + glob.glob(os.path.join(CSRC, "*.cpp")))


def _headers():
    return glob.glob(os.path.join(CSRC, "*.h")) + glob.glob(os.path.join(CSRC, "*.cuh")) + \
        glob.glob(os.path.join(HERE, "..", "include", "*.h"))


def _compile(src, verbose):
    obj = os.path.join(BUILD, os.path.basename(src) + ".o")
    newest_dep = max([os.path.getmtime(src)] + [os.path.getmtime(h) for h in _headers()])
    if os.path.exists(obj) and os.path.getmtime(obj) >= newest_dep:
        return obj
    cmd = [NVCC] + ARCH + FLAGS + ["-c", src, "-o", obj]
    if src.endswith(".cu"):
        cmd += ["-Xptxas", "-v"] if verbose else []
    else:
        cmd += ["-x", "cu"] if False else []
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"nvcc failed for {src}:\n{r.stdout}\n{r.stderr}")
    if verbose and r.stderr:
        sys.stderr.write(r.stderr)
    return obj


def _torch_dir():
    spec = importlib.util.find_spec("torch")  # found, not imported
    return os.path.dirname(spec.origin) if spec is not None and spec.origin else None


def _compile_bind_file(src):
    obj = os.path.join(BUILD, f"bind_{os.path.basename(src)[:-4]}.o")
    deps = [src] + glob.glob(os.path.join(BIND_DIR, "*.h")) + _headers()
    if os.path.exists(obj) and os.path.getmtime(obj) >= max(os.path.getmtime(f) for f in deps):
        return obj
    inc = [os.path.join(_torch_dir(), "include"), os.path.join(_torch_dir(), "include", "torch", "csrc", "api", "include"),
           sysconfig.get_paths()["include"], os.path.join(os.path.dirname(os.path.dirname(NVCC)), "include"),
           os.path.join(HERE, "..", "include")]
    cmd = ["g++", "-O2", "-std=c++20", "-fPIC", "-fvisibility=hidden", "-w", "-c", src, "-o", obj]
    r = subprocess.run(cmd + [x for i in inc for x in ("-I", i)], capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"g++ failed for {src}:\n{r.stdout}\n{r.stderr}")
    return obj


def _compile_bind():
    with cf.ThreadPoolExecutor() as ex:
        return list(ex.map(_compile_bind_file, sorted(glob.glob(os.path.join(BIND_DIR, "*.cpp")))))


def _link_bind(objs):
    if os.path.exists(BIND) and os.path.getmtime(BIND) >= max(os.path.getmtime(f) for f in objs + [LIB]):
        return
    cmd = ["g++", "-shared"] + objs + ["-o", BIND, "-L", os.path.join(_torch_dir(), "lib"), "-ltorch", "-ltorch_cpu", "-ltorch_python",
           "-lc10", "-lc10_cuda", "-L", HERE, "-l:libsn.so", "-Wl,-rpath,$ORIGIN"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stdout}\n{r.stderr}")


def build(verbose: bool = False, jobs: int | None = None) -> str:
    os.makedirs(BUILD, exist_ok=True)
    srcs = _sources()
    with cf.ThreadPoolExecutor(max_workers=jobs or min(16, os.cpu_count() or 4)) as ex:
        bind = ex.submit(_compile_bind) if _torch_dir() else None
        objs = list(ex.map(lambda s: _compile(s, verbose), srcs))
        _link(objs)  # first: what becomes of the front end does not touch the library
        if bind is not None:
            _link_bind(bind.result())
    return LIB


def _link(objs):
    if os.path.exists(LIB) and os.path.getmtime(LIB) >= max(os.path.getmtime(o) for o in objs):
        return
    cmd = [NVCC] + ARCH + ["-shared", "-o", LIB] + objs + ["-cudart", "static", "-lrt", "-ldl", "-lpthread"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stdout}\n{r.stderr}")


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
