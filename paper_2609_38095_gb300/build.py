"""Build libzo.so (the C-ABI library) in-tree for sm_103a.

Each .cu file is compiled by its own nvcc process (in parallel), then linked
into one shared library with the CUDA runtime linked statically; beside it the
Python module _binding.so (csrc/zo_binding.cpp) by the host compiler, which
alone needs torch.
Set ZO_PTXAS_VERBOSE=1 to print register / shared-memory usage.
"""
import concurrent.futures as cf
import importlib.metadata
import importlib.util
import os
import platform
import shutil
import subprocess
import sys
import sysconfig
import warnings

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(ROOT, "include")
BUILD = os.path.join(HERE, "_build", platform.machine())   # objects of this host architecture
LIB = os.path.join(HERE, "libzo.so")
BINDING = os.path.join(HERE, "_binding.so")   # the Python module of csrc/zo_binding.cpp
STAMP = LIB + ".arch"   # architecture the library was linked for
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
SOURCES = ["zo_api.cu", "zo_stream_kernels.cu", "zo_update_lut8.cu", "zo_small_kernels.cu",
           "zo_quad_step.cu", "zo_update_items.cu", "zo_update_blocks.cu",
           "zo_forward_api.cu", "zo_rotate.cu", "zo_attention.cu", "zo_attention_mma.cu",
           "zo_decode_mma.cu", "zo_decode_scalar.cu", "zo_token_loss.cu", "zo_answer_losses.cu", "zo_draft.cu", "zo_draft_wide.cu"]
HEADERS = ["zo_blocks.cuh", "zo_decode.cuh", "zo_device.cuh", "zo_forward.cuh", "zo_items.h", "zo_launch.h",
           "zo_logits.cuh", "zo_precond.cuh", "zo_tcgen05.cuh"]
ABI_HEADERS = ["zo.h", "zo_forward.h"]


def nvcc() -> str:
    p = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(p):
        raise RuntimeError("nvcc not found: the CUDA toolkit is required to build libzo.so")
    return p


def _flags():
    f = ["-O3", "-std=c++17", "-lineinfo", *ARCH, "-Xcompiler", "-fPIC", "-I", INCLUDE, "-I", CSRC]
    if os.environ.get("ZO_PTXAS_VERBOSE"):
        f += ["-Xptxas", "-v"]
    return f


def _binding_command(out):
    """One compiler call for the Python module, against the installed torch's headers and libraries."""
    torch = importlib.util.find_spec("torch")
    if torch is None:
        raise RuntimeError("torch not found: the Python module is built against it")
    torch = torch.submodule_search_locations[0]
    cuda = os.path.dirname(os.path.dirname(os.path.realpath(nvcc())))
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        raise RuntimeError("g++ not found: a C++ compiler is required to build the Python module")
    return [cxx, "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall", os.path.join(CSRC, "zo_binding.cpp"), "-o", out, "-I", INCLUDE,
            "-isystem", os.path.join(torch, "include"), "-isystem", sysconfig.get_path("include"), "-isystem",
            os.path.join(cuda, "include"), "-L", os.path.join(torch, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_cuda"]


def _torch_version():
    return importlib.metadata.version("torch")


def _stale(target, deps):
    if not os.path.exists(target):
        return True
    t = os.path.getmtime(target)
    return any(os.path.getmtime(d) > t for d in deps)


def _run(cmd):
    return cmd, subprocess.run(cmd, capture_output=True, text=True)


def build_binding(force: bool = False) -> str:
    """Build the Python module alone, against the installed torch; raises where that cannot be done, and leaves none
    that was built from other sources or for another torch."""
    try:
        made = f"{platform.machine()} {_torch_version()}"   # what it was built for
        ok = os.path.exists(BINDING + ".arch") and open(BINDING + ".arch").read().strip() == made
        deps = [os.path.join(CSRC, "zo_binding.cpp"), *(os.path.join(INCLUDE, h) for h in ABI_HEADERS), __file__]
        if not force and ok and not _stale(BINDING, deps):
            return BINDING
        tmp = BINDING + f".tmp{os.getpid()}"
        cmd, r = _run(_binding_command(tmp))
        if r.stdout or r.stderr:
            sys.stderr.write(r.stdout + r.stderr)
        if r.returncode != 0:
            raise RuntimeError(f"compiler failed: {' '.join(cmd)}")
        os.replace(tmp, BINDING)
        with open(BINDING + ".arch", "w") as f:
            f.write(made)
        return BINDING
    except Exception:
        for old in (BINDING, BINDING + ".arch"):
            if os.path.exists(old):
                os.remove(old)
        raise


def build(force: bool = False) -> str:
    """Build libzo.so, which needs no torch, and beside it the Python module of the forward point's operators. Where the
    latter cannot be built (a torch without headers, say) the library still is, with a warning; zo.forward's calls raise."""
    os.makedirs(BUILD, exist_ok=True)
    hdrs = [os.path.join(CSRC, h) for h in HEADERS] + [os.path.join(INCLUDE, h) for h in ABI_HEADERS]
    jobs = []
    objs = []
    for s in SOURCES:
        src = os.path.join(CSRC, s)
        obj = os.path.join(BUILD, s.replace(".cu", ".o"))
        objs.append(obj)
        if force or _stale(obj, [src] + hdrs + [__file__]):
            jobs.append([nvcc(), *_flags(), "-c", src, "-o", obj])

    with cf.ThreadPoolExecutor(max_workers=len(jobs) + 1) as ex:
        binding = ex.submit(build_binding, force)
        for cmd, r in ex.map(_run, jobs):
            if r.stdout or r.stderr:
                sys.stderr.write(r.stdout + r.stderr)
            if r.returncode != 0:
                raise RuntimeError(f"compiler failed: {' '.join(cmd)}")
    arch_ok = os.path.exists(STAMP) and open(STAMP).read().strip() == platform.machine()
    if force or jobs or not arch_ok or _stale(LIB, objs):
        tmp = LIB + f".tmp{os.getpid()}"
        cmd, r = _run([nvcc(), *ARCH, "-shared", "-cudart", "static", "-o", tmp, *objs])
        if r.returncode != 0:
            raise RuntimeError(f"link failed: {r.stderr}")
        os.replace(tmp, LIB)
        with open(STAMP, "w") as f:
            f.write(platform.machine())
    if binding.exception() is not None:
        warnings.warn(f"the Python module of the forward point's operators is not built: {binding.exception()}")
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv))
