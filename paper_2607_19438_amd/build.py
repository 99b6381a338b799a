"""Build the gfx950 shared library ``libqgemm.so`` in-tree with hipcc, and the Python binding's compiled part.

Usage: ``python -m paper_2607_19438_amd.build [--verbose]``.
"""
from __future__ import annotations

import hashlib
import os
import shutil
import subprocess
import sys
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libqgemm.so")
SOURCES = [os.path.join(CSRC, f) for f in ("qgemm_api.hip", "moe_direct.hip", "serve_api.hip", "step_api.hip")]
DEPS = SOURCES + [os.path.join(CSRC, f) for f in ("qgemm_kernels.hpp", "qgemm_aux.hpp", "qgemm_smallm.hpp", "moe_direct.hpp",
                                                  "moe_direct_api.hpp", "tile_rules.hpp", "attn_kernels.hpp", "api_util.hpp",
                                                  "serve_kernels.hpp", "attn_kv4.hpp", "kv4_levels.hpp", "attn_shared.hpp", "beam_kernels.hpp",
                                                  "adapter_kernels.hpp", "api_checks.hpp")] + [
    os.path.join(os.path.dirname(HERE), "include", "qgemm.h")]

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
ARCH = "gfx950"

FLAGS = [
    f"--offload-arch={ARCH}",
    "-O3",
    "-std=c++20",
    "-fPIC",
    # no packed-fp32 VALU instructions in any device code
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall",
    "-Wno-unused-command-line-argument",
]


HEADER = os.path.join(os.path.dirname(HERE), "include", "qgemm.h")


def header_stamp() -> str:
    """What the library and the binding each carry of the header that they were built from: a binding calls only a library
    of the same one."""
    with open(HEADER, "rb") as f:
        return hashlib.sha256(f.read()).hexdigest()[:16]


def build(verbose: bool = False, extra=None) -> str:
    """Compile every source (side by side, one object each) and link the library. All of it in a folder of
    its own beside the library, which then replaces the old one in one step: builds may run at once."""
    with tempfile.TemporaryDirectory(prefix="build-", dir=os.path.dirname(LIB)) as tmp:
        objs = [os.path.join(tmp, os.path.basename(src) + ".o") for src in SOURCES]
        new = os.path.join(tmp, os.path.basename(LIB))
        stamp = f'-DQGEMM_HEADER="{header_stamp()}"'
        cmds = [[HIPCC, *FLAGS, stamp, *(extra or []), "-c", src, "-o", obj] for src, obj in zip(SOURCES, objs)]
        link = [HIPCC, f"--offload-arch={ARCH}", "-shared", *objs, "-o", new]
        if verbose:
            for cmd in [*cmds, link]:
                print(" ".join(cmd), flush=True)
        procs = [subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True) for cmd in cmds]
        outs = [p.communicate()[0] for p in procs]
        rcs = [p.returncode for p in procs]
        if not any(rcs):
            res = subprocess.run(link, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
            outs.append(res.stdout)
            rcs.append(res.returncode)
        out = "\n".join(l for l in "".join(outs).splitlines() if "not a recognized feature" not in l)
        if any(rcs):
            raise RuntimeError(f"hipcc failed ({rcs}):\n{out}")
        if verbose and out.strip():
            print(out)
        os.replace(new, LIB)
    return LIB


BINDING = os.path.join(HERE, "_binding.so")
BINDING_SOURCE = os.path.join(CSRC, "binding.cpp")


def build_binding(verbose: bool = False):
    """Compile the host code between Python and the library (the serving calls' checks and allocations) against the
    installed torch; it replaces the old one in one step. Without a host compiler or Python's headers, which the library
    does not need, it is left unbuilt and None returned: the calls then go the Python way."""
    import sysconfig

    import torch
    compiler, include = os.environ.get("CXX", "g++"), sysconfig.get_paths()["include"]
    if shutil.which(compiler) is None or not os.path.exists(os.path.join(include, "Python.h")):
        print(f"{os.path.basename(BINDING)} not built: " + ("no Python.h" if shutil.which(compiler) else f"no {compiler}"), flush=True)
        return None
    root = os.path.join(os.path.dirname(torch.__file__))
    with tempfile.TemporaryDirectory(prefix="build-", dir=os.path.dirname(BINDING)) as tmp:
        new = os.path.join(tmp, os.path.basename(BINDING))
        cmd = [compiler, "-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden", "-Wall",
               f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", f'-DQGEMM_HEADER="{header_stamp()}"',
               f'-DQGEMM_TORCH="{torch.__version__}"', "-isystem", include,
               "-isystem", os.path.join(root, "include"), "-isystem", os.path.join(root, "include", "torch", "csrc", "api", "include"),
               BINDING_SOURCE, "-o", new, "-L" + os.path.join(root, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10"]
        if verbose:
            print(" ".join(cmd), flush=True)
        res = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
        if res.returncode:
            raise RuntimeError(f"{cmd[0]} failed ({res.returncode}):\n{res.stdout}")
        if verbose and res.stdout.strip():
            print(res.stdout)
        os.replace(new, BINDING)
    return BINDING


if __name__ == "__main__":
    v = "--verbose" in sys.argv
    extra = ["-Rpass-analysis=kernel-resource-usage"] if "--resources" in sys.argv else None
    print(build(verbose=v or bool(extra), extra=extra))
    if (binding := build_binding(verbose=v)) is not None:
        print(binding)
