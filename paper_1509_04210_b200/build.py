"""Builds ``librudra_ps.so`` in-tree with nvcc for sm_100a (cross-compiles without a GPU)."""
from __future__ import annotations

import hashlib
import importlib.metadata
import importlib.util
import os
import subprocess
import sys
import sysconfig

_PKG = os.path.dirname(os.path.abspath(__file__))
_CSRC = os.path.join(_PKG, "csrc")
_INCLUDE = os.path.join(os.path.dirname(_PKG), "include")
LIB_PATH = os.path.join(_PKG, "librudra_ps.so")
SOURCES = ["ps.cu", "update.cu", "snapshot.cu", "leaf.cu", "noalloc.cu", "sched.cpp",
           "learner.cu", "mx4.cu", "mx4_matmul.cu", "mx4_matmul_pair.cu", "act8.cu", "act8_weight_grad.cu",
           "fp8.cu", "fp8_matmul.cu", "fp8_matmul_pair.cu", "rms_norm.cu", "grad_clip.cu"]
# measurement utility of the benchmark, a library of its own: not part of the product interface
PROBE_LIB_PATH = os.path.join(_PKG, "librudra_probe.so")
PROBE_SOURCES = ["probe.cu"]
# the torch binding of the learner-side operators, host code only
LEARNER_PATH = os.path.join(_PKG, "_learner.so")
LEARNER_SOURCE = "learner_torch.cpp"
NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "-Xcompiler", "-fPIC", "-cudart", "static", "-shared", "-t", "0",
]


def _deps():
    out = [os.path.join(_CSRC, f) for f in os.listdir(_CSRC)]
    out += [os.path.join(_INCLUDE, f) for f in os.listdir(_INCLUDE)]
    return out


def needs_build(path: str = LIB_PATH) -> bool:
    if not os.path.exists(path):
        return True
    t = os.path.getmtime(path)
    return any(os.path.getmtime(d) > t for d in _deps())


def _compile(path, sources, verbose):
    nvcc = os.environ.get("NVCC", "nvcc")
    tmp = path + ".tmp.%d" % os.getpid()
    cmd = [nvcc] + NVCC_FLAGS + (["-Xptxas", "-v"] if verbose else []) + ["-I", _INCLUDE, "-o", tmp]
    cmd += os.environ.get("RUDRA_NVCC_DEFINES", "").split()   # e.g. "-DRUDRA_MID_THREADS=128" for a tile sweep
    cmd += [os.path.join(_CSRC, s) for s in sources]
    subprocess.check_call(cmd)
    os.replace(tmp, path)
    return path


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and not needs_build():
        return LIB_PATH
    return _compile(LIB_PATH, SOURCES, verbose)


def build_probe(force: bool = False, verbose: bool = False) -> str:
    if not force and not needs_build(PROBE_LIB_PATH):
        return PROBE_LIB_PATH
    return _compile(PROBE_LIB_PATH, PROBE_SOURCES, verbose)


def learner_sources() -> list:
    return [os.path.join(_CSRC, LEARNER_SOURCE), os.path.join(_INCLUDE, "rudra_learner.h"), os.path.join(_INCLUDE, "rudra_ps.h")]


def _torch_version() -> str:
    return importlib.metadata.version("torch")


def learner_key() -> str:
    """What a binding has to be built from: its sources, and the torch and Python it is loaded into.  Compiled into it."""
    h = hashlib.sha256()
    for path in learner_sources():
        with open(path, "rb") as f:
            h.update(f.read() + b"\0")
    h.update(("%s %s" % (_torch_version(), sysconfig.get_config_var("SOABI"))).encode())
    return h.hexdigest()


def learner_needs_build() -> bool:
    if not os.path.exists(LEARNER_PATH):
        return True
    with open(LEARNER_PATH, "rb") as f:
        return learner_key().encode() not in f.read()


def build_learner(force: bool = False) -> str:
    """The torch binding of the learner-side operators, a CPython module next to the library it calls."""
    if not force and not learner_needs_build():
        return LEARNER_PATH
    torch_dir = importlib.util.find_spec("torch").submodule_search_locations[0]
    cuda = os.environ.get("CUDA_HOME", "/usr/local/cuda")
    tmp = LEARNER_PATH + ".tmp.%d" % os.getpid()
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden", "-Wall",
           '-DRUDRA_LEARNER_KEY="%s"' % learner_key(),
           "-I", sysconfig.get_paths()["include"], "-I", _INCLUDE]
    for d in (os.path.join(torch_dir, "include"), os.path.join(torch_dir, "include", "torch", "csrc", "api", "include"), os.path.join(cuda, "include")):
        cmd += ["-isystem", d]
    cmd += [os.path.join(_CSRC, LEARNER_SOURCE), "-o", tmp, "-L", _PKG, "-l:" + os.path.basename(LIB_PATH), "-Wl,-rpath,$ORIGIN",
            "-L", os.path.join(torch_dir, "lib"), "-ltorch_python", "-ltorch_cuda", "-ltorch_cpu", "-lc10_cuda", "-lc10"]
    subprocess.check_call(cmd)
    os.replace(tmp, LEARNER_PATH)
    return LEARNER_PATH


def load_learner() -> None:
    """Builds the binding if it is absent or stale; a stale one is never loaded, its arguments may differ from the library's."""
    try:
        build_learner()
    except Exception as exc:
        raise ImportError("_learner.so is missing, or from other sources or another torch, and could not be built: %r" % (exc,)) from exc


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
    print(build_probe(force="--force" in sys.argv, verbose="-v" in sys.argv))
    print(build_learner(force="--force" in sys.argv))
