"""Builds in-tree: the CUDA library paper_2609_37447_b200/libazeval.so (nvcc, sm_100a only) and the binding's argument marshalling,
paper_2609_37447_b200/_tokens.so (g++, against the installed torch)."""
import glob
import hashlib
import importlib.metadata
import os
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libazeval.so")
BINDING = os.path.join(HERE, "_tokens.so")
STAMP = os.path.join(HERE, "build", "stamp.txt")
BINDING_STAMP = os.path.join(HERE, "build", "binding_stamp.txt")

NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xcompiler", "-fPIC", "--expt-relaxed-constexpr"]


def _hash(words, paths) -> str:
    h = hashlib.sha1(" ".join(words).encode())
    for path in sorted(paths):
        with open(path, "rb") as f:
            h.update(path.encode() + f.read())
    return h.hexdigest()


def _headers() -> list:
    return glob.glob(os.path.join(ROOT, "include", "*.h"))


def _digest() -> str:
    return _hash(NVCC_FLAGS, glob.glob(os.path.join(CSRC, "*.cu*")) + _headers())


def _binding_digest() -> str:
    return _hash([importlib.metadata.version("torch"), sys.version], [os.path.join(CSRC, "binding.cpp"), *_headers()])


def _current(built: str, stamp: str, digest: str) -> bool:
    return os.path.exists(built) and os.path.exists(stamp) and open(stamp).read().strip() == digest


def _binding_command() -> list:
    import torch
    root = os.path.dirname(torch.__file__)
    cuda = os.path.dirname(os.path.dirname(os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")))
    include = [os.path.join(ROOT, "include"), os.path.join(root, "include"), os.path.join(root, "include", "torch", "csrc", "api", "include"),
               os.path.join(cuda, "include"), sysconfig.get_paths()["include"]]
    return [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden",
            f"-D_GLIBCXX_USE_CXX11_ABI={int(torch.compiled_with_cxx11_abi())}",
            *(f"-I{i}" for i in include), os.path.join(CSRC, "binding.cpp"), "-o", BINDING,
            "-L" + os.path.join(root, "lib"), "-ltorch_python", "-ltorch", "-ltorch_cpu", "-lc10", "-lc10_cuda"]


def _build_library(verbose: bool, ptxas_info: bool):
    digest = _digest()
    if _current(LIB, STAMP, digest) and not ptxas_info:
        return
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    obj_dir = os.path.dirname(STAMP)
    os.makedirs(obj_dir, exist_ok=True)
    procs, objs = [], []
    for src in sorted(glob.glob(os.path.join(CSRC, "*.cu"))):
        obj = os.path.join(obj_dir, os.path.basename(src)[:-3] + ".o")
        objs.append(obj)
        cmd = [nvcc, *NVCC_FLAGS, "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-c", src, "-o", obj]
        if ptxas_info:
            cmd.insert(1, "-Xptxas=-v")
        procs.append((src, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    failed = False
    for src, p in procs:
        out, _ = p.communicate()
        if p.returncode != 0 or verbose or ptxas_info:
            sys.stderr.write(f"== {os.path.basename(src)}\n{out}\n")
        failed |= p.returncode != 0
    if failed:
        raise RuntimeError("nvcc failed")
    subprocess.run([nvcc, "-shared", "-o", LIB, *objs], check=True)
    with open(STAMP, "w") as f:
        f.write(digest)


def _build_binding(verbose: bool):
    digest = _binding_digest()
    if _current(BINDING, BINDING_STAMP, digest):
        return
    os.makedirs(os.path.dirname(BINDING_STAMP), exist_ok=True)
    p = subprocess.run(_binding_command(), stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    if p.returncode != 0 or verbose:
        sys.stderr.write(f"== binding.cpp\n{p.stdout}\n")
    if p.returncode != 0:
        raise RuntimeError(f"{os.environ.get('CXX', 'g++')} failed")
    with open(BINDING_STAMP, "w") as f:
        f.write(digest)


def build(verbose: bool = False, ptxas_info: bool = False) -> str:
    """Compile every .cu under csrc/ (in parallel) and link the shared library; then the binding of the token calls, without which the
    rest of the package works.  Returns the library's path."""
    _build_library(verbose, ptxas_info)
    try:
        _build_binding(verbose)
    except Exception as e:
        raise RuntimeError(f"{LIB} is built, the binding of the token calls is not: {e}") from e
    return LIB


if __name__ == "__main__":
    print(build(verbose=True, ptxas_info="--ptxas" in sys.argv))
