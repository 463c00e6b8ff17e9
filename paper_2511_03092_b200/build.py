"""Build libsnapstream.so (sm_100a only) in-tree with nvcc.

    python -m paper_2511_03092_b200.build [--force] [--verbose] [--debug-bounds]

Each csrc/*.cu is compiled to an object under csrc/build/ (in parallel, only when its
sources are newer) and the objects are linked into paper_2511_03092_b200/libsnapstream.so.
csrc/marshal.cpp becomes the extension module paper_2511_03092_b200/_marshal, which passes torch tensors to the
rotary and paged-cache entry points (it knows the library only by address).  It is built for one interpreter and one
torch: the file carries the interpreter's tag, the module the torch version, and either one's change builds it anew.
Without torch the library alone is built.
nvcc cross-compiles, so this works on a machine without a GPU.
--debug-bounds builds the checked variant instead (-DSNAP_DEBUG_BOUNDS: data-dependent indices are
tested and a bad one raises a status bit instead of an access; objects under csrc/build_dbg/) as
libsnapstream_dbg.so; the binding loads it when SNAP_LIBRARY names it.
"""
from __future__ import annotations

import glob
import importlib.util
import os
import shutil
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
OBJ = os.path.join(CSRC, "build")
LIB = os.path.join(PKG, "libsnapstream.so")
MARSHAL = os.path.join(PKG, "_marshal" + sysconfig.get_config_var("EXT_SUFFIX"))

ARCH = ["-gencode", "arch=compute_100a,code=sm_100a"]
COMMON = ["-O3", "-std=c++17", "-lineinfo", "-Xcompiler", "-fPIC",
          "-I", os.path.join(ROOT, "include"), "-I", CSRC]


def _nvcc() -> str:
    exe = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(exe):
        raise RuntimeError("nvcc not found; the CUDA toolkit is required to build libsnapstream")
    return exe


def _newest(paths) -> float:
    return max(os.path.getmtime(p) for p in paths)


def _built_for(path: str) -> str:
    """The torch version that a built module names, '' where there is none."""
    mark = b"built for torch "
    try:
        with open(path, "rb") as f:
            data = f.read()
    except OSError:
        return ""
    at = data.find(mark)
    return data[at + len(mark):data.index(b"\0", at)].decode() if at >= 0 else ""


def build_marshal(force: bool = False, verbose: bool = False) -> str:
    import torch
    src = os.path.join(CSRC, "marshal.cpp")
    torch_dir = os.path.dirname(torch.__file__)
    newest = _newest([src, os.path.join(ROOT, "include", "snapstream.h"), os.path.join(torch_dir, "version.py")])
    if not force and _built_for(MARSHAL) == str(torch.__version__) and os.path.getmtime(MARSHAL) >= newest:
        return MARSHAL
    cuda = os.path.dirname(os.path.dirname(os.path.realpath(_nvcc())))
    inc = [os.path.join(torch_dir, "include"), os.path.join(torch_dir, "include", "torch", "csrc", "api", "include"),
           sysconfig.get_paths()["include"], os.path.join(cuda, "include"), os.path.join(ROOT, "include")]
    lib = os.path.join(torch_dir, "lib")
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
           f'-DBUILT_FOR_TORCH="{torch.__version__}"', *[f"-isystem{d}" for d in inc[:-1]], "-I", inc[-1], src, "-o", MARSHAL, "-L", lib,
           "-lc10", "-lc10_cuda", "-ltorch_cpu", "-ltorch_python", f"-Wl,-rpath,{lib}"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if verbose or r.returncode != 0:
        sys.stderr.write(" ".join(cmd) + "\n" + r.stdout + r.stderr)
    if r.returncode != 0:
        raise RuntimeError("g++ failed for marshal.cpp")
    return MARSHAL


def build(force: bool = False, verbose: bool = False, debug_bounds: bool = False) -> str:
    obj_dir = OBJ + "_dbg" if debug_bounds else OBJ
    lib = os.path.join(PKG, "libsnapstream_dbg.so") if debug_bounds else LIB
    extra = ["-DSNAP_DEBUG_BOUNDS"] if debug_bounds else []
    os.makedirs(obj_dir, exist_ok=True)
    sources = sorted(glob.glob(os.path.join(CSRC, "*.cu")))
    headers = glob.glob(os.path.join(CSRC, "*.cuh")) + glob.glob(os.path.join(ROOT, "include", "*.h"))
    hdr_time = _newest(headers + [os.path.abspath(__file__)])
    nvcc = _nvcc()
    jobs = []
    objects = []
    for src in sources:
        obj = os.path.join(obj_dir, os.path.basename(src)[:-3] + ".o")
        objects.append(obj)
        if (not force and os.path.exists(obj)
                and os.path.getmtime(obj) >= max(os.path.getmtime(src), hdr_time)):
            continue
        cmd = [nvcc, *ARCH, *COMMON, *extra, "-c", src, "-o", obj]
        if verbose:
            cmd.insert(1, "-Xptxas=-v")
        jobs.append(cmd)

    def run(cmd):
        r = subprocess.run(cmd, capture_output=True, text=True)
        return cmd, r

    if jobs:
        with ThreadPoolExecutor(max_workers=min(8, len(jobs))) as ex:
            for cmd, r in ex.map(run, jobs):
                if verbose or r.returncode != 0:
                    sys.stderr.write(" ".join(cmd) + "\n" + r.stdout + r.stderr)
                if r.returncode != 0:
                    raise RuntimeError("nvcc failed for " + cmd[-3])
    if jobs or force or not os.path.exists(lib) or os.path.getmtime(lib) < _newest(objects):
        cmd = [nvcc, *ARCH, "-shared", "-o", lib, *objects]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            sys.stderr.write(r.stdout + r.stderr)
            raise RuntimeError("link failed")
    if importlib.util.find_spec("torch") is None:
        sys.stderr.write("torch is not installed: the library is built without the module that passes tensors to it\n")
    else:
        build_marshal(force and not debug_bounds, verbose)
    return lib


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="--verbose" in sys.argv, debug_bounds="--debug-bounds" in sys.argv))
