"""Builds libsilenzio_pbs.so (HIP, gfx950 only) in-tree with hipcc, and libsilenzio_torch.*.so, the binding's reader of tensor lists, with g++."""
from __future__ import annotations

import concurrent.futures
import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libsilenzio_pbs.so")
SOURCES = ["slz_api.hip", "slz_tables.hip", "slz_generic.hip", "slz_fft.hip", "slz_fft512.hip", "slz_fft1024.hip", "slz_fft2048.hip", "slz_fft2048_team.hip", "slz_fft2048_pair.hip", "slz_fft4096.hip", "slz_fft4096_pair.hip", "slz_fused_n512.hip", "slz_fused_n1024.hip", "slz_bign.hip", "slz_bign_xcd.hip", "slz_keyswitch.hip", "slz_keyswitch_mfma.hip",
           "slz_lincomb_mfma.hip", "slz_matmul_rns.hip", "slz_loss.hip",
           "slz_clear_common.hip", "slz_i8.hip", "slz_i4.hip", "slz_linear_ce.hip", "slz_orthogonalize.hip", "slz_clip.hip"]
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-ffp-contract=off", "-Wall", "-Wno-unused-function",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]


def _hipcc() -> str:
    for c in ("/opt/rocm/bin/hipcc", "hipcc"):
        if os.path.exists(c) or c == "hipcc":
            return c
    return "hipcc"


def _compile(src: str) -> str:
    obj = os.path.join(CSRC, "_build", src.replace(".hip", ".o"))
    os.makedirs(os.path.dirname(obj), exist_ok=True)
    cmd = [_hipcc(), *FLAGS, "-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    msgs = "\n".join(l for l in r.stdout.splitlines() if "packed-fp32-ops" not in l)
    if r.returncode != 0:
        raise RuntimeError("hipcc failed for %s:\n%s" % (src, msgs))
    if msgs.strip():
        print(msgs)
    return obj


def torch_lib() -> str:
    """The reader's path: it holds for one torch and one Python, which its name has."""
    import sys
    import torch
    return os.path.join(HERE, "libsilenzio_torch.%s.%s.so" % (torch.__version__.replace("+", "_"), sys.implementation.cache_tag))


def _build_tensors() -> None:
    import sysconfig
    import torch
    lib = torch_lib()
    at = os.path.dirname(torch.__file__)
    include = [os.path.join(at, "include"), os.path.join(at, "include", "torch", "csrc", "api", "include"), sysconfig.get_paths()["include"]]
    tmp = lib + ".tmp%d" % os.getpid()
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-w", "-D_GLIBCXX_USE_CXX11_ABI=%d" % torch._C._GLIBCXX_USE_CXX11_ABI, *("-I" + i for i in include),
           os.path.join(CSRC, "slz_tensors.cpp"), "-L" + os.path.join(at, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10", "-o", tmp]
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    if r.returncode != 0:
        raise RuntimeError("g++ failed for slz_tensors.cpp:\n%s" % r.stdout)
    os.replace(tmp, lib)


def build(verbose: bool = False) -> str:
    with concurrent.futures.ThreadPoolExecutor(max_workers=min(8, len(SOURCES))) as ex:
        tensors = ex.submit(_build_tensors)
        objs = list(ex.map(_compile, SOURCES))
    tmp = LIB + ".tmp%d" % os.getpid()
    subprocess.check_call([_hipcc(), "--offload-arch=gfx950", "-shared", "-fPIC", "-o", tmp, *objs])
    os.replace(tmp, LIB)
    tensors.result()                                   # after the library, which needs neither torch nor Python
    if verbose:
        print("built", LIB, torch_lib())
    return LIB


if __name__ == "__main__":
    build(verbose=True)
