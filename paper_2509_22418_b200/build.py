"""Builds libppu.so (sm_100a, nvcc) and _ops.so (the compiled torch binding of the operators, g++) next to this
file.  No GPU is needed to build.  The library needs neither torch nor the binding: where torch (with CUDA) is not
installed it is built alone, and where the binding does not compile the error comes once the library is there."""
from __future__ import annotations

import importlib.util
import os
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libppu.so")
OPS = os.path.join(HERE, "_ops.so")
SOURCES = ["ppu_api.cu", "ppu_step.cu", "elementwise.cu", "optim.cu", "gemm_simt.cu",
           "gemm_tc.cu", "gemm_tc_pair.cu", "attention_simt.cu", "attention_tc.cu", "attention_static.cu", "wait_probe.cu",
           "head_loss.cu", "norm_gate.cu", "embed.cu", "qk_norm.cu", "orthogonalize.cu"]
FLAGS = ["-O3", "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo",
         "-Xcompiler", "-fPIC", "--expt-relaxed-constexpr"]


def _stale() -> bool:
    built = [LIB, OPS] if _torch_dir() else [LIB]
    if not all(os.path.exists(p) for p in built):
        return True
    stamp = _stamp()
    if OPS in built and os.path.exists(stamp) and open(stamp).read() != _built_for():      # (without a note of it, the binding is taken as it is)
        return True
    t = min(os.path.getmtime(p) for p in built)
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC)]
    deps.append(os.path.join(os.path.dirname(HERE), "include", "ppu.h"))
    return any(os.path.getmtime(p) > t for p in deps)


OPS_OBJ = os.path.join(HERE, "_build", "bind.o")


def _torch_dir():
    """Where torch with CUDA is installed (found without importing it), or None."""
    spec = importlib.util.find_spec("torch")
    path = os.path.dirname(spec.origin) if spec and spec.origin else None
    return path if path and os.path.exists(os.path.join(path, "lib", "libtorch_cuda.so")) else None


def _stamp() -> str:
    return os.path.join(os.path.dirname(OPS_OBJ), "bind.txt")


def _built_for() -> str:
    """The torch and the Python that a binding belongs to: their ABI is not kept from one version to the next."""
    torch = _torch_dir()
    with open(os.path.join(torch, "version.py")) as f:
        return f"{sys.implementation.cache_tag}\n{torch}\n{f.read()}"


def _ops_compile():
    inc = os.path.join(_torch_dir(), "include")
    cuda = os.path.dirname(os.path.dirname(os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")))
    return ["g++", "-O2", "-std=c++17", "-fPIC", "-D_GLIBCXX_USE_CXX11_ABI=1", "-I" + inc, "-I" + os.path.join(inc, "torch", "csrc", "api", "include"),
            "-I" + sysconfig.get_paths()["include"], "-I" + os.path.join(cuda, "include"), "-c", os.path.join(CSRC, "bind.cpp"), "-o", OPS_OBJ]


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and not _stale():
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    objs, procs = [], []
    os.makedirs(os.path.join(HERE, "_build"), exist_ok=True)
    for src in SOURCES:
        obj = os.path.join(HERE, "_build", src.replace(".cu", ".o"))
        objs.append(obj)
        cmd = [nvcc, *FLAGS, "-c", os.path.join(CSRC, src), "-o", obj]
        if verbose:
            cmd.insert(1, "-Xptxas=-v")
        procs.append((src, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT)))
    with_ops, failed = _torch_dir() is not None, []
    if with_ops:
        try:
            procs.append(("bind.cpp", subprocess.Popen(_ops_compile(), stdout=subprocess.PIPE, stderr=subprocess.STDOUT)))
        except OSError as e:               # no such compiler
            sys.stderr.write(f"--- bind.cpp\n{e}\n")
            failed.append("bind.cpp")
    for src, p in procs:
        out = p.communicate()[0].decode()
        if p.returncode != 0 or verbose:
            sys.stderr.write(f"--- {src}\n{out}\n")
        if p.returncode != 0:
            failed.append(src)
    if [src for src in failed if src != "bind.cpp"]:
        raise RuntimeError(f"compilation failed: {', '.join(failed)}")
    subprocess.check_call([nvcc, "-shared", "-o", LIB, *objs, "-gencode",
                           "arch=compute_100a,code=sm_100a"])
    if not with_ops:
        sys.stderr.write("torch with CUDA is not installed: its binding (_ops.so) is not built\n")
        return LIB
    if failed:
        raise RuntimeError("compilation failed: bind.cpp")
    torch_lib = os.path.join(_torch_dir(), "lib")
    subprocess.check_call(["g++", "-shared", "-o", OPS, OPS_OBJ, "-L" + HERE, "-l:libppu.so", "-Wl,-rpath,$ORIGIN", "-L" + torch_lib, "-ltorch_python", "-ltorch",
                           "-ltorch_cpu", "-ltorch_cuda", "-lc10", "-lc10_cuda"])
    with open(_stamp(), "w") as f:
        f.write(_built_for())
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
