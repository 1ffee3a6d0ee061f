"""Builds liblynx.so (the HIP kernels and the C ABI) for gfx950, and _args.so (the
Python binding's test of a tensor argument, host code), in-tree.

hipcc flags: -O3, gfx950 only, no fast-math; packed-fp32 instructions are
disabled (-packed-fp32-ops) so the compiler never emits v_pk_{add,mul,fma}_f32.
"""
import os
import subprocess
import sys
import sysconfig
import warnings
from pathlib import Path

HERE = Path(__file__).resolve().parent
CSRC = HERE / "csrc"
ROOT = HERE.parent
LIBRARY = HERE / "liblynx.so"
ARGS = HERE / "_args.so"
SOURCES = ["codec.hip", "hier.hip", "attention.hip", "anchor_decode.hip", "anchor_split.hip", "verify.hip",
           "verify_wide.hip", "tree.hip", "append.hip", "spec.hip", "spec_tree.hip", "abi.hip"]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-fno-fast-math", "-Wall", "-Wno-unused-function",
    f"-I{ROOT / 'include'}", f"-I{CSRC}",
]


def _compile(cmd, target: Path, verbose: bool) -> Path:
    tmp = target.with_name(target.name + f".tmp{os.getpid()}")
    cmd = [*cmd, "-o", str(tmp)]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.run(cmd, check=True)
    os.replace(tmp, target)
    return target


def build_args(verbose: bool = False) -> Path:
    """Compile the binding's host code against this torch; always recompiles."""
    import torch

    home = Path(torch.__file__).parent
    return _compile(["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall",
                     f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
                     f"-isystem{home / 'include'}", f"-isystem{home / 'include/torch/csrc/api/include'}",
                     f"-isystem{sysconfig.get_paths()['include']}", str(CSRC / "host_args.cpp"), f"-L{home / 'lib'}",
                     "-ltorch_python", "-ltorch_cpu", "-lc10", f"-Wl,-rpath,{home / 'lib'}"], ARGS, verbose)


def build(verbose: bool = False) -> Path:
    """Compile every HIP source into liblynx.so, and the host code; always recompiles.
    The binding does without the host code: where that does not compile, a warning."""
    _compile([HIPCC, *FLAGS, *[str(CSRC / s) for s in SOURCES]], LIBRARY, verbose)
    try:
        build_args(verbose)
    except (OSError, subprocess.CalledProcessError) as e:  # no compiler, or not its headers
        ARGS.unlink(missing_ok=True)  # (an older one is not of these sources)
        warnings.warn(f"{ARGS.name} was not built ({e}): calls on trees, appends and read-back check their tensors in "
                      "Python, some 4 us more each")
    return LIBRARY


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
