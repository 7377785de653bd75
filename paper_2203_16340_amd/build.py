"""Builds liblbfgsb.so (the HIP kernels and their C-ABI) in-tree for gfx950, and _losses.so, the binding of the operators on logits to torch
tensors."""
from __future__ import annotations

import os
import subprocess
import sys
import sysconfig
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "liblbfgsb.so")
BINDING = os.path.join(HERE, "_losses.so")
SOURCES = ["fused.hip", "narrow.hip", "small.hip", "symmetric.hip", "gram.hip", "api.hip", "apass.hip", "resident.hip", "transport.hip", "vec.hip",
           "logits.hip", "logits_f32.hip", "logits_bf16.hip", "logits_f16.hip", "preference.hip", "losses_api.hip", "draws.hip", "weights4.hip", "matvec4_f32.hip", "matvec4_bf16.hip", "matvec4_f16.hip", "rollouts_api.hip"]
BINDING_SOURCES = ["losses_binding.cpp", "rollouts_binding.cpp"]
FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-fno-gpu-rdc",
    # packed-fp32 instructions are kept out of the generated code on purpose
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-command-line-argument", "-Wno-unknown-warning-option",
]


def build(verbose: bool = False, extra_flags=()) -> str:
    """One object per source, up to four at a time, then the shared library, then the binding (left out where torch or g++ is
    missing)."""
    with tempfile.TemporaryDirectory() as tmp:
        def compile_one(name: str) -> str:
            obj = os.path.join(tmp, name + ".o")
            cmd = ["hipcc", *FLAGS, *extra_flags, "-I", os.path.join(HERE, "..", "include"), "-c",
                   os.path.join(CSRC, name), "-o", obj]
            if verbose:
                print(" ".join(cmd), flush=True)
            subprocess.run(cmd, check=True)
            return obj

        with ThreadPoolExecutor(4) as pool:
            binding = [pool.submit(compile_binding, name, os.path.join(tmp, name + ".o"), verbose) for name in BINDING_SOURCES]
            objects = list(pool.map(compile_one, SOURCES))
        subprocess.run(["hipcc", "--offload-arch=gfx950", "-shared", "-fPIC", *objects, "-o", LIB], check=True)
        # The library, which needs neither torch nor g++, is there from here on, whatever becomes of the binding (an older one does
        # not go with it).
        if os.path.exists(BINDING):
            os.remove(BINDING)
        try:
            link_binding([b.result() for b in binding], verbose)
        except (ImportError, FileNotFoundError) as e:
            print(f"{BINDING} is not built, and the losses on logits not callable from Python: {e}", file=sys.stderr, flush=True)
    return LIB


def compile_binding(name: str, obj: str, verbose: bool = False) -> str:
    """Host code only: torch's headers, no device code."""
    import torch
    from torch.utils import cpp_extension
    include = [*cpp_extension.include_paths(), sysconfig.get_paths()["include"]]
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-DTORCH_EXTENSION_NAME=_losses",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", *(a for i in include for a in ("-isystem", i)),
           "-c", os.path.join(CSRC, name), "-o", obj]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.run(cmd, check=True)
    return obj


def link_binding(objects, verbose: bool = False) -> str:
    """Against liblbfgsb.so beside it and torch's libraries, which are loaded before it."""
    from torch.utils import cpp_extension
    cmd = ["g++", "-shared", *objects, "-o", BINDING, "-L" + HERE, "-l:liblbfgsb.so", *("-L" + d for d in cpp_extension.library_paths()),
           "-ltorch", "-ltorch_cpu", "-ltorch_python", "-lc10", "-Wl,-rpath,$ORIGIN"]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.run(cmd, check=True)
    return BINDING


if __name__ == "__main__":
    build(verbose=True, extra_flags=sys.argv[1:])
