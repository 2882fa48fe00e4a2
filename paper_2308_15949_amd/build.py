"""Builds liblaud.so (gfx950 HIP kernels + C ABI) in-tree with hipcc, and _laud_torch.so, the extension that calls the token
operators from torch tensors, with the host compiler.

    python -m paper_2308_15949_amd.build

The library needs hipcc only: where torch cannot be imported the extension is left out, with a line on stderr, and where it does not
compile the library is there before the error is raised.

Every source is compiled to an object of its own (in parallel), then linked; objects live in
csrc/_build/ (ignored by git).
"""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
OBJ = os.path.join(CSRC, "_build")
LIB = os.path.join(HERE, "liblaud.so")
EXTENSION = os.path.join(HERE, "_laud_torch.so")
SOURCES = ["laud_api.hip", "laud_mask.hip", "laud_chanmask.hip", "laud_static.hip", "laud_se.hip", "laud_gemm.hip", "laud_pipe_a.hip", "laud_pipe_b.hip", "laud_pipe_c.hip", "laud_group.hip", "laud_group_fused.hip", "laud_skinny.hip", "laud_narrow.hip", "laud_first.hip",
           "laud_probe.hip", "laud_tail.hip", "laud_head.hip", "laud_norm.hip", "laud_matmul8.hip", "laud_moe.hip"]
# packed-fp32 code generation is switched off for device code (the host pass warns that it
# does not know the feature; that is harmless).
FLAGS = ["-O3", "-std=c++17", "--offload-arch=gfx950", "-fPIC",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-I", os.path.join(ROOT, "include"), "-I", CSRC]


def _run(cmd, verbose):
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, capture_output=True, text=True)
    err = "\n".join(l for l in res.stderr.splitlines() if "is not a recognized feature" not in l)
    if res.returncode != 0:
        sys.stderr.write(err + "\n")
        raise RuntimeError(os.path.basename(cmd[0]) + " failed: " + " ".join(cmd[-3:]))
    if verbose and err.strip():
        print(err)


def extension_command() -> list[str]:
    """The host compiler's command for _laud_torch.so (host code only: Python, torch and HIP runtime headers)."""
    import sysconfig

    import torch
    home = os.path.dirname(torch.__file__)
    include = [os.path.join(home, "include"), os.path.join(home, "include", "torch", "csrc", "api", "include"),
               os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "include")]
    return [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-shared", "-fPIC", "-D__HIP_PLATFORM_AMD__=1", "-DUSE_ROCM=1",
            f"-D_GLIBCXX_USE_CXX11_ABI={int(torch.compiled_with_cxx11_abi())}",
            "-I", os.path.join(ROOT, "include"), "-I", sysconfig.get_paths()["include"],
            *(a for d in include for a in ("-isystem", d)), os.path.join(CSRC, "laud_torch.cpp"), "-o", EXTENSION,
            "-L", os.path.join(home, "lib"), "-lc10", "-lc10_hip", "-ltorch_cpu", "-ltorch_python"]


def build(verbose: bool = True) -> str:
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    os.makedirs(OBJ, exist_ok=True)
    objs = [os.path.join(OBJ, s.replace(".hip", ".o")) for s in SOURCES]
    jobs = [[hipcc, *FLAGS, "-c", os.path.join(CSRC, s), "-o", o] for s, o in zip(SOURCES, objs)]
    try:
        extension = extension_command()
    except ImportError as e:
        extension = None
        sys.stderr.write(f"{os.path.basename(EXTENSION)} (calls of the token operators from torch tensors) is left out: {e}\n")
    with ThreadPoolExecutor(max_workers=min(8, len(jobs) + 1)) as ex:
        made = ex.submit(_run, extension, verbose) if extension else None
        list(ex.map(lambda c: _run(c, verbose), jobs))
    _run([hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", *objs, "-o", LIB], verbose)
    if made:
        made.result()  # (raises what the extension's compiler said, behind the library's link)
    return LIB


if __name__ == "__main__":
    print(build())
