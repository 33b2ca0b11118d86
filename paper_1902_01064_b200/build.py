"""Compiles csrc/ into libhop_b200.so (in-tree, next to this file) with nvcc for sm_100a, and the host side of the layer
operators on torch tensors into _hop_nn.so with g++."""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libhop_b200.so")
LIB_CHECKED = os.path.join(HERE, "libhop_b200_checked.so")      # same sources with -DHOP_CHECKED (tests only)
SOURCES = ["hop_api.cu", "hop_kernels.cu", "hop_dense_tc.cu", "hop_static.cu", "hop_norm.cu", "hop_norm_f32.cu", "hop_norm_f16.cu",
           "hop_norm_bf16.cu", "hop_linear.cu", "hop_sim.cpp", "hop_trace.cpp"]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found")


NN_LIB = os.path.join(HERE, "_hop_nn.so")
NN_SOURCE = "hop_nn_torch.cpp"


def _torch_dir() -> str | None:
    import importlib.util
    spec = importlib.util.find_spec("torch")
    return os.path.dirname(spec.origin) if spec else None


def _build_nn(verbose: bool) -> None:
    import sysconfig
    torch_dir = _torch_dir()
    cuda = os.path.dirname(os.path.dirname(os.path.realpath(_nvcc())))
    # the system's g++, whose libstdc++ torch is linked to as well (a second, static one in this module breaks its streams and
    # exceptions; $CXX may be a toolchain of that kind)
    cmd = [shutil.which("g++") or "c++", "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall", os.path.join(CSRC, NN_SOURCE), "-o", NN_LIB,
           "-I", os.path.join(ROOT, "include"), "-isystem", os.path.join(torch_dir, "include"), "-isystem", os.path.join(torch_dir, "include/torch/csrc/api/include"),
           "-isystem", os.path.join(cuda, "include"), "-isystem", sysconfig.get_paths()["include"],
           "-L", os.path.join(torch_dir, "lib"), "-lc10", "-lc10_cuda", "-ltorch_cpu", "-ltorch_python", "-Wl,-rpath," + os.path.join(torch_dir, "lib")]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if verbose or r.returncode != 0:
        sys.stderr.write(r.stdout + r.stderr)
    if r.returncode != 0:
        raise RuntimeError("g++ failed building " + os.path.basename(NN_LIB))


def needs_build(lib: str = LIB) -> bool:
    made = [lib] + ([NN_LIB] if lib == LIB and _torch_dir() else [])
    if not all(os.path.exists(m) for m in made):
        return True
    t = min(os.path.getmtime(m) for m in made)
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC)] + [os.path.join(ROOT, "include", "hop.h")]
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = False, verbose: bool = False, checked: bool = False) -> str:
    """checked=True builds libhop_b200_checked.so: every global-memory source of a bulk copy or cp.async of the mix kernels and
    every SVM gather is tested against the bound buffers first (select it with HOP_B200_LIBRARY=<path> before importing hop).
    The layer operators bind no buffers; they are the same in both."""
    lib = LIB_CHECKED if checked else LIB
    if not force and not needs_build(lib):
        return lib
    flags = ["-O3", "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-Xcompiler", "-fPIC",
             "-I", os.path.join(ROOT, "include"), "-I", CSRC] + (["-DHOP_CHECKED"] if checked else []) + (["-Xptxas", "-v"] if verbose else [])

    def run(cmd):
        r = subprocess.run(cmd, capture_output=True, text=True)
        if verbose or r.returncode != 0:
            sys.stderr.write(r.stdout + r.stderr)
        if r.returncode != 0:
            raise RuntimeError("nvcc failed building " + os.path.basename(lib))

    with tempfile.TemporaryDirectory() as tmp:      # one nvcc per source, side by side
        objects = [os.path.join(tmp, s + ".o") for s in SOURCES]
        with ThreadPoolExecutor((os.cpu_count() or 4) + 1) as pool:
            nn = pool.submit(_build_nn, verbose) if not checked and _torch_dir() else None
            list(pool.map(lambda so: run([_nvcc(), *flags, "-c", os.path.join(CSRC, so[0]), "-o", so[1]]), zip(SOURCES, objects)))
        run([_nvcc(), "-gencode", "arch=compute_100a,code=sm_100a", "-shared", "-o", lib, *objects])
    if nn is not None:
        nn.result()         # (the library, which needs neither torch nor g++, is there by now)
    elif not checked:
        sys.stderr.write("torch is not installed: " + os.path.basename(NN_LIB) + " (the layer operators on torch tensors) is left out\n")
    return lib


if __name__ == "__main__":
    print(build(force=True, verbose="-v" in sys.argv, checked="--checked" in sys.argv))
