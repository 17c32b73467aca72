"""Compile the HIP library in-tree for gfx950 (cross-compiles without a GPU), and the host extension of the torch class."""
from __future__ import annotations

import os
import subprocess
import sysconfig
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
SRC = os.path.join(HERE, "csrc", "lasgd.hip")
LAYERS_SRC = os.path.join(HERE, "csrc", "lasgd_layers.hip")
LIB = os.path.join(HERE, "liblasgd_hip.so")
WALK_SRC = os.path.join(HERE, "csrc", "grad_walk.cpp")
WALK_LIB = os.path.join(HERE, "_grad_walk" + sysconfig.get_config_var("EXT_SUFFIX"))     # another Python does not load it

FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17",
    "-ffp-contract=off",                      # only the written fmaf calls fuse
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-fPIC", "-shared", "-Wall", "-Wno-unused-function",
]


def build_hip(verbose: bool = False) -> str:
    """Both translation units at the same time, then the library."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    with tempfile.TemporaryDirectory() as d:
        objs = [os.path.join(d, f"{i}.o") for i in range(2)]
        cmds = [[hipcc] + [f for f in FLAGS if f != "-shared"] + ["-c", "-o", o, src] for o, src in zip(objs, (SRC, LAYERS_SRC))]
        link = [hipcc, "--offload-arch=gfx950", "-fPIC", "-shared", "-o", LIB, *objs]
        if verbose:
            print("\n".join(" ".join(c) for c in (*cmds, link)), flush=True)
        running = [subprocess.Popen(c) for c in cmds]
        for code, c in zip([r.wait() for r in running], cmds):
            if code:
                raise subprocess.CalledProcessError(code, c)
        subprocess.check_call(link)
    return LIB


def build_grad_walk(verbose: bool = False) -> str:
    """Host code against the installed torch's headers and libraries."""
    import torch
    root = os.path.dirname(torch.__file__)
    inc = [os.path.join(root, "include"), os.path.join(root, "include", "torch", "csrc", "api", "include"),
           sysconfig.get_paths()["include"]]
    lib = os.path.join(root, "lib")
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
           f'-DLASGD_TORCH_VERSION="{torch.__version__}"', *["-isystem" + d for d in inc], "-o", WALK_LIB, WALK_SRC, "-L" + lib, "-ltorch_python", "-ltorch_cpu", "-lc10",
           "-Wl,-rpath," + lib]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.check_call(cmd)
    return WALK_LIB


if __name__ == "__main__":
    print(build_hip(verbose=True))
    print(build_grad_walk(verbose=True))
