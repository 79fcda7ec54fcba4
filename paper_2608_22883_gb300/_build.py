"""Build libfovea.so (the C-ABI library) in-tree for sm_103a with nvcc, and beside
it fovea_binding.so, the Python module of the drafter's cache.

Each translation unit under csrc/ is compiled in parallel, then linked into
``paper_2608_22883_gb300/_lib/libfovea.so`` (the CUDA ones) and
``_lib/fovea_binding.so`` (binding.cpp, with torch's headers and the host
compiler; without a torch with CUDA it is left out).  Objects go to ``_build/`` at the
repository root.  All of it is git-ignored.
"""

from __future__ import annotations

import concurrent.futures
import importlib.util
import os
import shutil
import subprocess
import sys
import sysconfig

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
BUILD = os.path.join(ROOT, "_build")
LIBDIR = os.path.join(PKG, "_lib")
LIB = os.path.join(LIBDIR, "libfovea.so")
BINDING = os.path.join(LIBDIR, "fovea_binding.so")

ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
CFLAGS = ["-O3", "-std=c++17", "-lineinfo", "-Xcompiler", "-fPIC,-fvisibility=hidden",
          "-I", INCLUDE, "-I", CSRC]


def nvcc() -> str:
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found: the CUDA toolkit is required to build libfovea")


def cxx() -> str:
    found = os.environ.get("CXX") or shutil.which("g++")
    if not found:
        raise RuntimeError("no host compiler: set CXX, or put g++ on the path")
    return found


def sources():
    return sorted(os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".cu"))


def torch_home():
    """The folder of the torch with CUDA that is installed, None without one (it is not imported)."""
    spec = importlib.util.find_spec("torch")
    home = "" if spec is None else os.path.dirname(spec.origin)
    return home if os.path.exists(os.path.join(home, "lib", "libc10_cuda.so")) else None


def binding_flags(home):
    """(flags to compile binding.cpp, flags to link it) against the torch in this folder."""
    cuda = os.path.dirname(os.path.dirname(nvcc()))
    compile_flags = ["-O2", "-std=c++17", "-fPIC", "-fvisibility=hidden", "-I", INCLUDE, "-isystem", os.path.join(home, "include"),
                     "-isystem", os.path.join(home, "include", "torch", "csrc", "api", "include"),
                     "-isystem", os.path.join(cuda, "include"), "-isystem", sysconfig.get_paths()["include"]]
    link_flags = ["-L", LIBDIR, "-lfovea", "-Wl,-rpath,$ORIGIN", "-L", os.path.join(home, "lib"), "-ltorch_python",
                  "-ltorch_cuda", "-ltorch_cpu", "-lc10_cuda", "-lc10"]
    return compile_flags, link_flags


def _newer(out: str, deps) -> bool:
    if not os.path.exists(out):
        return False
    t = os.path.getmtime(out)
    return all(os.path.getmtime(d) <= t for d in deps)


def _read(path: str):
    if not os.path.exists(path):
        return None
    with open(path) as f:
        return f.read()


def build(verbose: bool = False, force: bool = False, extra_flags=()) -> str:
    """Compile and link libfovea.so, and fovea_binding.so where there is a torch;
    returns the library's path.  Rebuilds only what changed (any header change
    rebuilds every object)."""
    os.makedirs(BUILD, exist_ok=True)
    os.makedirs(LIBDIR, exist_ok=True)
    cc = nvcc()
    headers = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".cuh", ".h"))]
    headers += [os.path.join(INCLUDE, f) for f in os.listdir(INCLUDE)]
    headers.append(os.path.abspath(__file__))
    jobs = []
    objs = []
    for src in sources():
        obj = os.path.join(BUILD, os.path.basename(src)[:-3] + ".o")
        objs.append(obj)
        if force or not _newer(obj, [src] + headers):
            jobs.append([cc, *ARCH, *CFLAGS, *extra_flags, "-c", src, "-o", obj])

    note, made_with = os.path.join(BUILD, "binding.txt"), None
    links = [(LIB, objs, [cc, *ARCH, "-shared", "-o", LIB, *objs, "-lpthread", "-ldl", "-lrt"])]
    home = torch_home()
    if home is not None:
        compile_flags, link_flags = binding_flags(home)
        host = cxx()
        source, binding = os.path.join(CSRC, "binding.cpp"), os.path.join(BUILD, "binding.o")
        cmd = [host, *compile_flags, "-c", source, "-o", binding]
        # made with this command against this torch: another one's objects do not go with its libraries
        with open(os.path.join(home, "version.py")) as f:
            made_with = " ".join(cmd) + "\n" + f.read()
        if force or _read(note) != made_with or not _newer(binding, [source] + headers):
            if os.path.exists(note):
                os.remove(note)
            jobs.insert(0, cmd)      # first: it takes as long as the longest of the others
        links.append((BINDING, [binding, LIB], [host, "-shared", "-o", BINDING, binding, *link_flags]))

    def run(cmd):
        r = subprocess.run(cmd, capture_output=True, text=True)
        return cmd, r

    if jobs:
        with concurrent.futures.ThreadPoolExecutor(max_workers=min(len(jobs), os.cpu_count() or 4)) as ex:
            for cmd, r in ex.map(run, jobs):
                if verbose or r.returncode != 0:
                    sys.stderr.write(" ".join(cmd) + "\n" + r.stdout + r.stderr)
                if r.returncode != 0:
                    raise RuntimeError(f"{os.path.basename(cmd[0])} failed on {cmd[-3]}")
    if made_with is not None and _read(note) != made_with:
        with open(note, "w") as f:
            f.write(made_with)
    for out, parts, cmd in links:
        if not force and not jobs and _newer(out, parts):
            continue
        _, r = run(cmd)
        if verbose or r.returncode != 0:
            sys.stderr.write(" ".join(cmd) + "\n" + r.stdout + r.stderr)
        if r.returncode != 0:
            raise RuntimeError(f"linking {os.path.basename(out)} failed")
    return LIB


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv, force="-f" in sys.argv))
