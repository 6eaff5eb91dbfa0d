"""Builds libzkdl.so (the C-ABI HIP library) for gfx950 with hipcc, and _layers8.so (Python's side of its 8-bit layers), in-tree."""
import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
OUT = os.path.join(HERE, "libzkdl.so")
SOURCES = ["api.hip", "k_basic.hip", "k_sumcheck.hip", "k_scpair.hip", "k_schelp.hip", "k_zkrelu.hip", "k_zkprefix.hip", "k_zkshort.hip", "k_zkhelp.hip", "k_zktail.hip", "k_reindex.hip", "k_selfbench.hip", "k_commit.hip", "k_verify.hip", "k_general.hip", "k_layer8.hip", "k_matmul8.hip"]
FLAGS = ["-O3", "-std=c++17", "--offload-arch=gfx950", "-fPIC", "-fno-gpu-rdc",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-Wno-unused-command-line-argument", "-Wno-unknown-attributes"]


def _compile(src):
    obj = os.path.join(HERE, "_build", src.replace(".hip", ".o"))
    cmd = ["hipcc", *FLAGS, "-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    return src, obj, r


MODULE = os.path.join(HERE, "_layers8.so")      # Python's side of the 8-bit layers, against the installed torch


def _module_command():
    """The compiler's command for the module, or why there is none: it needs torch with its headers and g++, which the C library does not."""
    import shutil
    import sysconfig
    try:
        import torch
        from torch.utils import cpp_extension
    except ImportError as e:
        return None, f"torch cannot be imported ({e})"
    paths = cpp_extension.include_paths() + [sysconfig.get_paths()["include"], "/opt/rocm/include"]
    for header in ("torch/csrc/autograd/python_variable.h", "Python.h"):
        if not any(os.path.exists(os.path.join(d, header)) for d in paths):
            return None, f"{header} is not installed"
    if not shutil.which("g++"):
        return None, "g++ is not installed"
    lib = os.path.join(os.path.dirname(torch.__file__), "lib")
    return ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-w", "-D__HIP_PLATFORM_AMD__=1", "-DUSE_ROCM=1",
            f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", *[f"-I{d}" for d in paths], os.path.join(CSRC, "layers8_torch.cpp"),
            "-o", MODULE, f"-L{lib}", f"-Wl,-rpath,{lib}", "-lc10", "-lc10_hip", "-ltorch_cpu", "-ltorch_hip", "-ltorch_python"], ""


def _module():
    """Compiles the module; returns the compiler's result and, where there was nothing to run, why."""
    if os.path.exists(MODULE):
        os.remove(MODULE)       # one that is older than its source would be taken for this one
    cmd, why = _module_command()
    return (subprocess.run(cmd, capture_output=True, text=True) if cmd else None), why


def build(verbose=True):
    """Compiles and links libzkdl.so, then tells what became of the module: the prover is there whether or not that could be made, and the
    8-bit layers raise ImportError without it."""
    os.makedirs(os.path.join(HERE, "_build"), exist_ok=True)
    with ThreadPoolExecutor(max_workers=8) as ex:
        pending = ex.submit(_module)
        results = list(ex.map(_compile, SOURCES))
        module, why = pending.result()
    objs = []
    for src, obj, r in results:
        if r.returncode != 0:
            sys.stderr.write(r.stdout + r.stderr)
            raise RuntimeError(f"hipcc failed on {src}")
        if verbose and r.stderr.strip():
            errs = [l for l in r.stderr.splitlines() if "packed-fp32-ops" not in l and l.strip()]
            if errs:
                sys.stderr.write("\n".join(errs) + "\n")
        objs.append(obj)
    r = subprocess.run(["hipcc", "--offload-arch=gfx950", "-shared", "-fPIC", *objs, "-o", OUT],
                       capture_output=True, text=True)
    if r.returncode != 0:
        sys.stderr.write(r.stdout + r.stderr)
        raise RuntimeError("link failed")
    if module is None:
        sys.stderr.write(f"_layers8.so is not built, the 8-bit layers will be missing from Python: {why}\n")
    elif module.returncode != 0:
        sys.stderr.write(module.stdout + module.stderr)
        raise RuntimeError("g++ failed on layers8_torch.cpp (libzkdl.so is built)")
    return OUT


if __name__ == "__main__":
    print(build())
