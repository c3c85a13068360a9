"""Build libhpf.so (the C-ABI CUDA library) in-tree with nvcc for sm_100a, and _calls (argument marshalling for Python) with the C compiler.

The library is all that is needed.  _calls is an extension of the interpreter that builds it, which its file name tells; without
Python's headers or a C compiler the binding marshals by ctypes.
"""
import os
import subprocess
import sys
import sysconfig
import warnings

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libhpf.so")
CALLS = os.path.join(HERE, "_calls" + (sysconfig.get_config_var("EXT_SUFFIX") or ".so"))
CALLS_SOURCE = os.path.join(CSRC, "py_calls.c")
HEADER = os.path.join(HERE, "..", "include", "hpf.h")
SOURCES = ["hpf_model.cu", "kernels_mem.cu", "conv_simt.cu", "conv_tc.cu", "conv_pipe.cu", "no_alloc.cu", "bn_resident.cu", "logprobs.cu", "distill.cu", "linear.cu"]
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-lineinfo", "-std=c++17",
              "-Xcompiler", "-fPIC", "-Xcompiler", "-Wall", "--use_fast_math=false"]


def _sources():
    return [os.path.join(CSRC, s) for s in SOURCES if os.path.exists(os.path.join(CSRC, s))]


def _older(path, deps):
    if not os.path.exists(path):
        return True
    t = os.path.getmtime(path)
    return any(os.path.getmtime(d) > t for d in deps)


def _stale():
    return _older(LIB, [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f != os.path.basename(CALLS_SOURCE)] + [HEADER])


def calls(force: bool = False):
    """The path of _calls, compiled if it is older than its sources; None (and a warning) where it cannot be."""
    if not force and not _older(CALLS, [CALLS_SOURCE, HEADER]):
        return CALLS
    made = f"{CALLS}.{os.getpid()}"                       # several processes may come here at once
    cmd = [os.environ.get("CC", "gcc"), "-O2", "-Wall", "-shared", "-fPIC", "-I", sysconfig.get_paths()["include"], CALLS_SOURCE, "-o", made]
    try:
        subprocess.run(cmd, check=True, capture_output=True, text=True)
        os.replace(made, CALLS)
    except (OSError, subprocess.CalledProcessError) as e:
        warnings.warn(f"{os.path.basename(CALLS)} could not be compiled, calls are marshalled by ctypes: {(getattr(e, 'stderr', None) or str(e)).strip()[:300]}")
        return None
    return CALLS


def build(force: bool = False, verbose: bool = False) -> str:
    if force or _stale():
        _build_library(verbose)
    calls(force)
    return LIB


def _build_library(verbose):
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    objs = []
    procs = []
    for src in _sources():
        obj = os.path.join(CSRC, os.path.basename(src)[:-3] + ".o")
        extra = os.environ.get("HPF_NVCC_EXTRA", "").split()          # e.g. -DHPF_RES_TIMELINE for latency studies
        cmd = [nvcc] + [f for f in NVCC_FLAGS if not f.startswith("--use_fast_math")] + extra + (["-Xptxas", "-v"] if verbose else []) + ["-c", src, "-o", obj]
        procs.append((cmd, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
        objs.append(obj)
    for cmd, p in procs:
        out, _ = p.communicate()
        if verbose or p.returncode:
            sys.stderr.write(out)
        if p.returncode:
            raise RuntimeError("nvcc failed: " + " ".join(cmd))
    link = [nvcc, "-shared", "-o", LIB] + objs + ["-lcudart"]
    subprocess.run(link, check=True)


if __name__ == "__main__":
    print(build(force=True, verbose="-v" in sys.argv))
