"""Build the CUDA library in-tree: nvcc, sm_100a only, one shared object next to this file; and, where torch is installed, the
operators' binding for its tensors beside it.  A caller of the C entry points needs the first alone."""
from __future__ import annotations

import importlib.util
import os
import shutil
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
LIB = os.path.join(HERE, "libasd_b200.so")
SOURCES = ["asd_api.cu", "asd_kernels.cu", "asd_resident.cu", "asd_gemm.cu", "asd_mlp_fused.cu", "asd_static.cu", "asd_schedule.cu",
           "asd_ops_api.cu", "asd_ops_rows.cu", "asd_ops_gemm.cu", "asd_ops_stream.cu", "asd_ops_split.cu"]


TORCH_LIB = os.path.join(HERE, "_asd_torch.so")  # the operators for torch tensors


def _build_torch_binding(force: bool) -> None:
    """csrc/asd_torch.cpp against this environment's torch, next to the library it calls; without torch there is none."""
    if importlib.util.find_spec("torch") is None:
        return
    import sysconfig
    import torch
    src = os.path.join(HERE, "csrc", "asd_torch.cpp")
    # what it was built for: the interfaces of torch and Python change from version to version
    built, this = os.path.splitext(TORCH_LIB)[0] + ".built", f"torch {torch.__version__}, Python {sysconfig.get_python_version()}\n"
    if not force and os.path.exists(TORCH_LIB) and os.path.getmtime(TORCH_LIB) >= _newest([src, os.path.join(ROOT, "include", "asd_ops.h")]) and \
            os.path.exists(built) and open(built).read() == this:
        return
    from torch.utils import cpp_extension as ext
    libs = os.path.join(os.path.dirname(torch.__file__), "lib")
    cmd = [shutil.which("g++") or "g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-w",
           "-D_GLIBCXX_USE_CXX11_ABI=%d" % int(torch.compiled_with_cxx11_abi()), "-DTORCH_EXTENSION_NAME=_asd_torch", "-DTORCH_API_INCLUDE_EXTENSION_H",
           "-I" + os.path.join(ROOT, "include"), "-I" + sysconfig.get_paths()["include"]]
    cmd += ["-I" + p for p in ext.include_paths("cuda")]
    cmd += [src, "-o", TORCH_LIB, "-L" + HERE, "-l:libasd_b200.so", "-Wl,-rpath,$ORIGIN", "-L" + libs, "-Wl,-rpath," + libs,
            "-lc10", "-lc10_cuda", "-ltorch_cpu", "-ltorch_cuda", "-ltorch", "-ltorch_python"]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("the C library is built; g++ failed on its torch binding, " + src + ":\n" + res.stdout + res.stderr)
    with open(built, "w") as f:
        f.write(this)


def _newest(paths):
    return max(os.path.getmtime(p) for p in paths)


def build(force: bool = False, verbose: bool = False) -> str:
    srcs = [os.path.join(HERE, "csrc", s) for s in SOURCES]
    deps = srcs + [os.path.join(HERE, "csrc", "asd_internal.h"), os.path.join(HERE, "csrc", "asd_device.cuh"),
                   os.path.join(HERE, "csrc", "asd_tc.cuh"),
                   os.path.join(HERE, "csrc", "asd_ops_internal.h"), os.path.join(HERE, "csrc", "asd_ops_tc.cuh"),
                   os.path.join(HERE, "csrc", "asd_ops_act.cuh"),
                   os.path.join(ROOT, "include", "asd.h"), os.path.join(ROOT, "include", "asd_ops.h")]
    if not force and os.path.exists(LIB) and os.path.getmtime(LIB) >= _newest(deps):
        _build_torch_binding(force)
        return LIB
    nvcc = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    flags = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17", "-Xcompiler", "-fPIC",
             "-I" + os.path.join(ROOT, "include")]
    if verbose:
        flags.append("-Xptxas=-v")
    # one object per translation unit, compiled side by side (no device code is linked across them)
    obj_dir = os.path.join(HERE, "_build")
    os.makedirs(obj_dir, exist_ok=True)
    hdr_time = _newest(deps[len(srcs):])
    jobs = []
    for src in srcs:
        obj = os.path.join(obj_dir, os.path.basename(src)[:-3] + ".o")
        if force or verbose or not os.path.exists(obj) or os.path.getmtime(obj) < max(os.path.getmtime(src), hdr_time):
            jobs.append((src, subprocess.Popen([nvcc] + flags + ["-c", src, "-o", obj], stdout=subprocess.PIPE,
                                               stderr=subprocess.STDOUT, text=True)))
    log = []
    for src, proc in jobs:
        out, _ = proc.communicate()
        log.append(out)
        if proc.returncode != 0:
            raise RuntimeError("nvcc failed on " + src + ":\n" + out)
    objs = [os.path.join(obj_dir, os.path.basename(src)[:-3] + ".o") for src in srcs]
    res = subprocess.run([nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-shared", "-cudart", "static", "-o", LIB] + objs,
                         capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("link failed:\n" + res.stdout + res.stderr)
    _build_torch_binding(force)
    if verbose:
        print("".join(log))
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
