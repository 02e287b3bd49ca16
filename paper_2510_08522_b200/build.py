"""In-tree build of the shared objects (nvcc, sm_100a only):
    lib/libdmx.so          the gradient-step library (C ABI of include/dmx.h)
    lib/libdmx_gen.so      the synthetic-input fill kernels
    lib/libdmx_checked.so  (with --checked) the gradient-step library compiled with -DDMX_DEBUG:
                           every index into the tables and the scratch is range-tested on the
                           device; a violation sets DMX_FLAG_BOUNDS in the state vector, never a trap
Run as `python -m paper_2510_08522_b200.build [--force] [--verbose] [--checked]`.
"""
from __future__ import annotations

import os
import subprocess
import sys

_PKG = os.path.dirname(os.path.abspath(__file__))
_ROOT = os.path.dirname(_PKG)
CSRC = os.path.join(_PKG, "csrc")
LIBDIR = os.path.join(_PKG, "lib")
INCLUDE = os.path.join(_ROOT, "include")

NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xcompiler", "-fPIC", "-I", INCLUDE, "-I", CSRC]

TARGETS = {
    "libdmx.so": (["dmx.cu", "dmx_static.cu", "dmx_agg.cu", "dmx_ctl.cu", "dmx_adamw.cu", "dmx_group_norm.cu", "dmx_linear.cu"],
                  ["dmx_kernels.cuh", "dmx_act.cuh", "dmx_f32x2.cuh", "dmx_host.h", os.path.join(INCLUDE, "dmx.h")]),
    "libdmx_gen.so": (["dmx_gen.cu"], []),
}


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if cand and (os.path.isabs(cand) and os.path.exists(cand) or not os.path.isabs(cand)):
            return cand
    return "nvcc"


TORCH_MODULE = "_dmx_torch.so"


def _torch_command():
    """g++ for the torch module. Its undefined symbols are those of the torch libraries that `import torch` has loaded."""
    import importlib.util
    import sysconfig
    torch = importlib.util.find_spec("torch").submodule_search_locations[0]
    cuda = os.path.join(os.path.dirname(os.path.dirname(_nvcc())), "include") if os.path.isabs(_nvcc()) else "/usr/local/cuda/include"
    inc = [os.path.join(torch, "include"), os.path.join(torch, "include", "torch", "csrc", "api", "include"), sysconfig.get_paths()["include"], cuda, INCLUDE]
    return (["g++", "-std=c++17", "-O2", "-fPIC", "-shared", "-fvisibility=hidden", "-Wno-attributes"] + ["-isystem" + i for i in inc[:-1]] + ["-I", INCLUDE] +
            [os.path.join(CSRC, "dmx_torch.cpp"), "-L", os.path.join(torch, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_cuda"])


def _newer(path: str, than: list) -> bool:
    """path exists and is at least as new as every file of `than`."""
    return os.path.exists(path) and all(os.path.getmtime(path) >= os.path.getmtime(d) for d in than)


def lib_path(name: str) -> str:
    return os.path.join(LIBDIR, name)


CHECKED = {"libdmx_checked.so": TARGETS["libdmx.so"]}


def build(force: bool = False, verbose: bool = False, checked: bool = False) -> None:
    """Bring the targets up to date: every source file is compiled to an object of its own (lib/_build/),
    the missing and the stale ones side by side, and the objects are linked. (dmx.cu alone takes about a
    minute and a half.)"""
    from concurrent.futures import ThreadPoolExecutor
    os.makedirs(LIBDIR, exist_ok=True)
    targets = dict(TARGETS)
    if checked:
        targets.update(CHECKED)
    compiles, links = [], []
    for name, (srcs, deps) in targets.items():
        out = lib_path(name)
        deps_abs = [d if os.path.isabs(d) else os.path.join(CSRC, d) for d in deps]
        objs, stale = [], False
        for src in (os.path.join(CSRC, s) for s in srcs):
            obj = os.path.join(LIBDIR, "_build", "%s.%s.o" % (name[:-3], os.path.basename(src)))
            objs.append(obj)
            if force or not _newer(obj, [src] + deps_abs):
                stale = True
                flags = NVCC_FLAGS + (["-DDMX_DEBUG"] if name in CHECKED else []) + (["-Xptxas", "-v"] if verbose else [])
                compiles.append(([_nvcc()] + flags + ["-c", src], obj))
        if stale or not _newer(out, objs):
            links.append(([_nvcc()] + NVCC_FLAGS + ["-shared"] + objs, out))

    out = lib_path(TORCH_MODULE)
    if force or not _newer(out, [os.path.join(CSRC, "dmx_torch.cpp"), os.path.join(INCLUDE, "dmx.h")]):
        compiles.append((_torch_command(), out))

    def run(job):
        cmd, out = job
        tmp = "%s.%d.tmp" % (out, os.getpid())
        cmd = cmd + ["-o", tmp]
        if verbose:
            print(" ".join(cmd), flush=True)
        subprocess.check_call(cmd)
        os.replace(tmp, out)

    for jobs in (compiles, links):
        if jobs:
            os.makedirs(os.path.join(LIBDIR, "_build"), exist_ok=True)
            # verbose: one at a time, which keeps ptxas' output in order
            with ThreadPoolExecutor(max_workers=1 if verbose else min(len(jobs), os.cpu_count() or 1)) as pool:
                for _ in pool.map(run, jobs):       # re-raises the first failure
                    pass


if __name__ == "__main__":
    build(force="--force" in sys.argv, verbose="--verbose" in sys.argv, checked="--checked" in sys.argv)
