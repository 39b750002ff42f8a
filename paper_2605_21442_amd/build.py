"""Build liblce.so in-tree for gfx950 with hipcc, and the Python extension _tensors (no JIT cache, no setup.py)."""
from __future__ import annotations

import os
import subprocess
import sys
import sysconfig

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
SRC = os.path.join(PKG, "csrc", "lce.hip")
OUT = os.path.join(PKG, "liblce.so")
TENSORS_SRC = os.path.join(PKG, "csrc", "tensors.cpp")
TENSORS_OUT = os.path.join(PKG, "_tensors" + sysconfig.get_config_var("EXT_SUFFIX"))   # (no other interpreter loads it)
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
CXX = os.environ.get("CXX", "g++")
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")

FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared",
    "-I", os.path.join(ROOT, "include"),
    # packed fp32 instructions stay off (hipcc's host pass warns that it does not know the feature)
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
]


def _run(cmd: list[str], out: str, verbose: bool) -> None:
    tmp = out + ".tmp"
    res = subprocess.run([*cmd, "-o", tmp], capture_output=True, text=True)
    if res.returncode != 0:
        sys.stderr.write(res.stdout + res.stderr)
        raise RuntimeError(f"{os.path.basename(cmd[0])} failed ({res.returncode}): {' '.join(cmd)}")
    if verbose:
        sys.stderr.write(res.stderr)
    os.replace(tmp, out)


def build_tensors(verbose: bool = False) -> str:
    """The host extension, against the installed torch (whose libraries are in the process before it is loaded)."""
    import torch
    from torch.utils import cpp_extension

    lib = os.path.join(os.path.dirname(torch.__file__), "lib")
    include = [f"-I{p}" for p in (*cpp_extension.include_paths(), sysconfig.get_paths()["include"])]
    _run([CXX, "-O2", "-std=c++17", "-fPIC", "-shared", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch.compiled_with_cxx11_abi())}",
          "-D__HIP_PLATFORM_AMD__=1", "-DUSE_ROCM=1", *include, f"-I{os.path.join(ROCM, 'include')}", TENSORS_SRC,
          f"-L{lib}", "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_hip"], TENSORS_OUT, verbose)
    return TENSORS_OUT


def build(verbose: bool = False) -> str:
    _run([HIPCC, *FLAGS, SRC], OUT, verbose)
    build_tensors(verbose)
    return OUT


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
