"""Builds libmlora.so (sm_100a only) next to this file with nvcc, and with the host compiler the module that checks and hands on the
tensors of its cache operators.  No JIT cache: both stay in-tree."""
import importlib.metadata
import importlib.util
import os
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
SOURCES = ["w4_gemm.cu", "lora_shrink.cu", "step_misc.cu", "attention.cu", "decode_chain.cu", "decode_step.cu", "decode_lean.cu", "w4_gemm_tc.cu", "attn_tc.cu", "w4a8_gemm.cu", "rope.cu", "attn_scored.cu", "kv_evict.cu", "mlora.cu"]
LIB = os.path.join(HERE, "libmlora.so")
MARSHAL = os.path.join(HERE, "_marshal.so")
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xcompiler", "-fPIC"]


def _newer(target, deps):
    if not os.path.exists(target):
        return False
    t = os.path.getmtime(target)
    return all(os.path.getmtime(d) <= t for d in deps)


def build(force=False, verbose=False):
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    headers = [os.path.join(CSRC, "common.cuh"), os.path.join(CSRC, "pipe.cuh"), os.path.join(CSRC, "tc.cuh"), os.path.join(CSRC, "cache_ops.cuh"), os.path.join(HERE, "..", "include", "mlora.h")]
    objdir = os.path.join(HERE, "_build")
    os.makedirs(objdir, exist_ok=True)
    objs = []
    procs = []
    for s in SOURCES:
        src = os.path.join(CSRC, s)
        obj = os.path.join(objdir, s.replace(".cu", ".o"))
        objs.append(obj)
        if not force and _newer(obj, [src] + headers):
            continue
        cmd = [nvcc] + NVCC_FLAGS + (["-Xptxas", "-v"] if verbose else []) + ["-c", src, "-o", obj]
        procs.append((cmd, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    for cmd, p in procs:
        out, _ = p.communicate()
        if verbose or p.returncode:
            sys.stderr.write(out)
        if p.returncode:
            raise RuntimeError("nvcc failed: " + " ".join(cmd))
    if force or procs or not _newer(LIB, objs):
        cmd = [nvcc, "-shared", "-gencode", "arch=compute_100a,code=sm_100a", "-o", LIB] + objs + ["-lcudart"]
        subprocess.check_call(cmd)
    build_marshal(force, verbose)
    return LIB


def _marshal_made_for():
    """The torch and Python that `_marshal.so` is compiled against; None where there is no torch"""
    spec = importlib.util.find_spec("torch")
    if spec is None:
        return None
    try:
        version = importlib.metadata.version("torch")
    except importlib.metadata.PackageNotFoundError:        # a source tree on the path
        version = str(os.path.getmtime(spec.origin))
    return f"{spec.origin} {version} {sys.implementation.cache_tag}\n"


def build_marshal(force=False, verbose=False):
    """The module that hands on the tensors of the cache operators, after the library, which does not need it.  Made again when its
    sources, torch or Python change; left out where there is no torch (then nothing can import the binding either)."""
    made_for = _marshal_made_for()
    if made_for is None:
        return
    src, stamp = os.path.join(CSRC, "marshal.cpp"), MARSHAL + ".made_for"
    if not force and _newer(MARSHAL, [src, os.path.join(HERE, "..", "include", "mlora.h")]) and os.path.exists(stamp):
        with open(stamp) as f:
            if f.read() == made_for:
                return
    import torch
    root = os.path.dirname(torch.__file__)
    cuda = os.path.dirname(os.path.dirname(os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")))
    inc = [os.path.join(root, "include"), os.path.join(root, "include", "torch", "csrc", "api", "include"), sysconfig.get_paths()["include"],
           os.path.join(cuda, "include")]
    lib = os.path.join(root, "lib")
    cmd = ([os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}"] +
           ["-isystem" + d for d in inc] + [src, "-o", MARSHAL, "-L" + lib, "-Wl,-rpath," + lib, "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_cuda"])
    try:
        done = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
        out, code = done.stdout, done.returncode
    except OSError as e:
        out, code = f"{e}\n", 1
    if verbose or code:
        sys.stderr.write(out)
    if code:
        raise RuntimeError("libmlora.so is built, _marshal.so (the binding's calls around a bounded KV cache) is not: " + " ".join(cmd))
    with open(stamp, "w") as f:
        f.write(made_for)


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
