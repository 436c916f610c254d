"""Build libffint8.so (HIP, gfx950 only) in-tree with hipcc.

    python -m paper_2506_22771_amd.build [--force]

and _bind.so, the compiled marshalling of Python's calls on matrices of floating-point values: norms, checkpoints, gated layers, dropout (host code, against Python's and torch's
headers), with g++.
Where one of these is not there the library is built all the same, for its C interface and the other Python calls; what is missing is printed.

-ffp-contract=off: the numerics need one rounding per written fp32 operation (hipcc would fuse).
-packed-fp32-ops is switched off as required on the test machines."""
from __future__ import annotations

import concurrent.futures as cf
import importlib.util
import os
import shutil
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
OBJ_DIR = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libffint8.so")
BIND = os.path.join(HERE, "_bind.so")
SOURCES = ["elementwise.hip", "gemm_i8.hip", "gemm_few.hip", "conv.hip", "conv3.hip", "conv3_wide.hip", "wgrad3.hip", "rows.hip", "fused.hip", "api.hip",
           "norm.hip", "ckpt.hip", "ckpt_wgrad.hip", "api_norm.hip", "gated.hip", "gated_grad.hip", "group_norm.hip", "group_norm_f32.hip", "group_norm_bf16.hip", "group_norm_f16.hip", "dropout.hip", "api_blocks.hip"]
HEADERS = [os.path.join(CSRC, "ff_internal.hpp"), os.path.join(CSRC, "device_math.hpp"), os.path.join(CSRC, "codes.hpp"), os.path.join(CSRC, "window.hpp"), os.path.join(CSRC, "ckpt.hpp"),
           os.path.join(CSRC, "act.hpp"), os.path.join(CSRC, "chunks.hpp"), os.path.join(CSRC, "norm.hpp"), os.path.join(CSRC, "norm_math.hpp"), os.path.join(CSRC, "api_checks.hpp"),
           os.path.join(CSRC, "blocks.hpp"), os.path.join(CSRC, "group_norm.hpp"), os.path.join(CSRC, "group_norm_forward.hpp"), os.path.join(CSRC, "group_norm_backward.hpp"), os.path.join(CSRC, "group_norm_plan.hpp"), os.path.join(CSRC, "wgrad_plan.hpp"), os.path.join(os.path.dirname(HERE), "include", "ffint8.h")]
FLAGS = ["--offload-arch=gfx950", "-O3", "-fPIC", "-std=c++17", "-ffp-contract=off", "-fno-fast-math",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-Wall", "-Wno-unused-function", "-Wno-inline-asm"]


def _stale(target: str, deps) -> bool:
    if not os.path.exists(target):
        return True
    t = os.path.getmtime(target)
    return any(os.path.getmtime(d) > t for d in deps)


def _compile(src: str, force: bool) -> str:
    obj = os.path.join(OBJ_DIR, os.path.splitext(src)[0] + ".o")
    path = os.path.join(CSRC, src)
    if force or _stale(obj, [path] + HEADERS):
        subprocess.run(["hipcc", *FLAGS, "-c", path, "-o", obj], check=True)
    return obj


def _bind_needs() -> dict:
    """What building _bind.so takes, and where it is (None: not there)."""
    spec = importlib.util.find_spec("torch")   # (without importing it)
    torch = os.path.join(os.path.dirname(spec.origin), "include") if spec and spec.origin else None
    python = sysconfig.get_paths()["include"]
    return {"g++": shutil.which("g++"), "Python's headers": python if os.path.exists(os.path.join(python, "Python.h")) else None,
            "torch's headers": torch if torch and os.path.exists(os.path.join(torch, "torch", "csrc", "autograd", "python_variable.h")) else None}


def _build_bind(force: bool) -> None:
    src = os.path.join(CSRC, "bind.cpp")
    if not (force or _stale(BIND, [src, LIB, HEADERS[-1]])):
        return
    needs = _bind_needs()
    missing = [what for what, where in needs.items() if where is None]
    if missing:
        if os.path.exists(BIND):
            os.remove(BIND)     # (it is older than the library)
        print(f"_bind.so is not built ({', '.join(missing)} not found): no calls of norms, checkpoints, gated layers and dropout from Python", file=sys.stderr)
        return
    torch = needs["torch's headers"]
    subprocess.run([needs["g++"], "-O2", "-fPIC", "-shared", "-std=c++17", "-Wall", "-D_GLIBCXX_USE_CXX11_ABI=1", "-I" + torch, "-I" + os.path.join(torch, "torch", "csrc", "api", "include"),
                    "-I" + needs["Python's headers"], src, "-o", BIND + ".tmp", "-L" + os.path.join(os.path.dirname(torch), "lib"),
                    "-ltorch_python", "-ltorch_cpu", "-lc10", "-L" + HERE, "-l:libffint8.so", "-Wl,-rpath,$ORIGIN"], check=True)
    os.replace(BIND + ".tmp", BIND)


def build(force: bool = False) -> str:
    os.makedirs(OBJ_DIR, exist_ok=True)
    with cf.ThreadPoolExecutor(max_workers=len(SOURCES)) as ex:
        objs = list(ex.map(lambda s: _compile(s, force), SOURCES))
    if force or _stale(LIB, objs):
        subprocess.run(["hipcc", "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB + ".tmp", *objs], check=True)
        os.replace(LIB + ".tmp", LIB)
    _build_bind(force)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv))
