"""Build libdflare.so (HIP, gfx950) and the native part of the Python binding (_binding.so) in-tree, in
paper_2606_02091_amd/_lib/."""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIBDIR = os.path.join(PKG, "_lib")
LIB = os.path.join(LIBDIR, "libdflare.so")
BINDING = os.path.join(LIBDIR, "_binding.so")
SOURCES = ["kernels.hip", "batched.hip", "runtime.hip", "training.hip", "train_ops.hip",
           "linear_ce.hip", "linear.hip", "qk_norm.hip", "adamw.hip"]
ARCH = os.environ.get("DFLARE_OFFLOAD_ARCH", "gfx950")


def hipcc() -> str:
    for cand in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", shutil.which("hipcc")):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("hipcc not found")


def build(verbose: bool = False) -> str:
    """Compile every HIP source of the library for gfx950 and link the shared object; beside it the binding's native part.
    The library needs neither PyTorch nor Python's headers: it is in its place before a binding that cannot be built
    raises BindingError (and takes an older binding with it)."""
    os.makedirs(LIBDIR, exist_ok=True)
    common = [f"--offload-arch={ARCH}", "-O3", "-std=c++17", "-fPIC",
              # keep the compiler away from packed fp32 instructions
              "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
              "-I", INCLUDE, "-I", CSRC, "-Wall", "-Wno-unused-function"]
    objs = [os.path.join(LIBDIR, src.replace(".hip", ".o")) for src in SOURCES]
    cmds = [[hipcc(), *common, "-c", os.path.join(CSRC, src), "-o", obj]
            for src, obj in zip(SOURCES, objs)]
    # the translation units are independent: compile them side by side
    with ThreadPoolExecutor(max_workers=len(cmds) + 1) as ex:
        units = [ex.submit(_run, cmd, verbose) for cmd in cmds]
        binding = BINDING + f".tmp{os.getpid()}"
        part = ex.submit(lambda: _run(_binding_command(binding), verbose))
        for f in units:
            f.result()
        tmp = LIB + f".tmp{os.getpid()}"
        _run([hipcc(), f"--offload-arch={ARCH}", "-shared", "-fPIC", *objs, "-o", tmp], verbose)
        os.replace(tmp, LIB)
        for o in objs:
            os.remove(o)
        try:
            part.result()
            os.replace(binding, BINDING)
        except Exception as e:
            if os.path.exists(BINDING):
                os.remove(BINDING)  # (it may call the new library with an older one's arguments)
            raise BindingError(f"{LIB} is built without {os.path.basename(BINDING)}: {e}") from e
    return LIB


class BindingError(RuntimeError):
    """The library is built; the native part of the Python binding is not."""


def _binding_command(out: str) -> list[str]:
    """The host compiler's command for the binding's native part (CPython and PyTorch C++ API, no GPU code)."""
    import torch
    from torch.utils import cpp_extension
    libs = os.path.join(os.path.dirname(torch.__file__), "lib")
    return ["g++", "-O2", "-std=c++17", "-shared", "-fPIC",
            f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", "-I", INCLUDE,
            *(f"-I{p}" for p in cpp_extension.include_paths()), f"-I{sysconfig.get_paths()['include']}",
            os.path.join(CSRC, "binding.cpp"), "-o", out, f"-L{libs}", "-ltorch_python", "-ltorch_cpu", "-lc10"]


def _run(cmd, verbose):
    if verbose:
        print(" ".join(cmd), flush=True)
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    out = "\n".join(l for l in r.stdout.splitlines() if "packed-fp32-ops" not in l)
    if r.returncode != 0:
        raise RuntimeError(f"build failed ({r.returncode}):\n{out}")
    if verbose and out.strip():
        print(out)


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
