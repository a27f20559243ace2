"""Build libacdc.so (HIP, gfx950) in-tree with hipcc, and the native part of the
training operators' binding (_train_binding.so) with the host compiler.

Usage: python -m paper_1511_05946_amd.build   (or build() from Python)
"""

from __future__ import annotations

import os
import shutil
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIB = os.path.join(PKG, "libacdc.so")
BINDING = os.path.join(PKG, "_train_binding.so")

# -packed-fp32-ops: keep every fp32 operation a plain VOP (no v_pk_*_f32).
HIP_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++20", "-fPIC",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wno-unused-command-line-argument",
]


def source_digest() -> str:
    """sha256 over the cascade's kernel sources (csrc/*, include/*), in name
    order: the version tag that recorded profiler counters are tied to.  The
    training operators' files (acdc_train*) are not in it: no cascade kernel
    includes them."""
    import hashlib
    h = hashlib.sha256()
    for d in (CSRC, INCLUDE):
        for name in sorted(os.listdir(d)):
            path = os.path.join(d, name)
            if os.path.isfile(path) and not name.startswith("acdc_train"):
                h.update(name.encode())
                with open(path, "rb") as f:
                    h.update(f.read())
    return h.hexdigest()


def hipcc() -> str:
    for cand in (os.environ.get("HIPCC"), shutil.which("hipcc"), "/opt/rocm/bin/hipcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("hipcc not found")


def build(verbose: bool = False, extra_flags: list[str] | None = None) -> str:
    """libacdc.so and, where the host has what that takes, the binding's native
    part against it.  The library and its C ABI need hipcc alone."""
    build_library(verbose, extra_flags)
    missing = missing_for_binding()
    if missing is None:
        build_binding(verbose)
    else:
        if os.path.exists(BINDING):
            os.remove(BINDING)   # an older library's
        sys.stderr.write(f"no {missing}: {os.path.basename(BINDING)} is not built, which losses and optim need\n")
    return LIB


def build_library(verbose: bool = False, extra_flags: list[str] | None = None) -> str:
    """Compile every csrc/*.hip to an object (in parallel), then link libacdc.so."""
    import tempfile
    srcs = sorted(os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".hip"))
    with tempfile.TemporaryDirectory(prefix="acdc_build_") as tmpdir:
        objs, procs = [], []
        for src in srcs:
            obj = os.path.join(tmpdir, os.path.basename(src) + ".o")
            cmd = [hipcc(), *HIP_FLAGS, *(extra_flags or []), "-I", INCLUDE, "-I", CSRC, "-c", src, "-o", obj]
            if verbose:
                print(" ".join(cmd), flush=True)
            procs.append((src, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.PIPE, text=True)))
            objs.append(obj)
        failed = False
        for src, proc in procs:
            out, err = proc.communicate()
            if proc.returncode != 0:
                sys.stderr.write(out + err)
                failed = True
        if failed:
            raise RuntimeError("hipcc failed")
        tmp = LIB + ".tmp"
        cmd = [hipcc(), "--offload-arch=gfx950", "-fPIC", "-shared", *objs, "-o", tmp]
        if verbose:
            print(" ".join(cmd), flush=True)
        proc = subprocess.run(cmd, capture_output=True, text=True)
        if proc.returncode != 0:
            sys.stderr.write(proc.stdout + proc.stderr)
            raise RuntimeError(f"hipcc link failed ({proc.returncode})")
        os.replace(tmp, LIB)
    return LIB


def host_compiler() -> str | None:
    return shutil.which(os.environ.get("CXX", "g++"))


def missing_for_binding() -> str | None:
    """What this host lacks for the binding's native part."""
    import importlib.util
    import sysconfig
    if host_compiler() is None:
        return "host C++ compiler (g++)"
    if not os.path.exists(os.path.join(sysconfig.get_paths()["include"], "Python.h")):
        return "Python.h"
    return None if importlib.util.find_spec("torch") is not None else "torch"


def build_binding(verbose: bool = False) -> str:
    """Compile csrc/acdc_train_binding.cpp against torch and libacdc.so."""
    import sysconfig

    import torch
    from torch.utils.cpp_extension import include_paths
    missing, cxx = missing_for_binding(), host_compiler()
    if missing is not None:
        raise RuntimeError(f"no {missing} found")
    includes = [a for p in (*include_paths(), sysconfig.get_paths()["include"]) for a in ("-isystem", p)]
    tmp = BINDING + ".tmp"
    cmd = [cxx, "-O2", "-std=c++17", "-fPIC", "-shared", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
           *includes, "-I", INCLUDE, os.path.join(CSRC, "acdc_train_binding.cpp"), "-o", tmp,
           "-L", os.path.join(os.path.dirname(torch.__file__), "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10",
           "-L", PKG, "-l:libacdc.so", "-Wl,-rpath,$ORIGIN"]
    if verbose:
        print(" ".join(cmd), flush=True)
    proc = subprocess.run(cmd, capture_output=True, text=True)
    if proc.returncode != 0:
        sys.stderr.write(proc.stdout + proc.stderr)
        raise RuntimeError(f"{cxx} failed ({proc.returncode})")
    os.replace(tmp, BINDING)
    return BINDING


if __name__ == "__main__":
    print(build(verbose=True))
