"""Builds libaq.so (CUDA, sm_100a only) next to this file with nvcc, and _aq_torch.so (its calls on torch tensors) with the host compiler.

    python -m paper_2605_24011_b200.build [--force]

libaq.so wants nvcc alone.  _aq_torch.so wants torch, g++ and Python's headers besides; where one of them is missing it is left out, with a
line on stderr, and the calls that go through it say so when they are made.

Objects go to paper_2605_24011_b200/_build/ (kept out of version control).
"""
from __future__ import annotations

import concurrent.futures
import os
import shutil
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
OUT = os.path.join(HERE, "libaq.so")
TORCH_OUT = os.path.join(HERE, "_aq_torch.so")
OBJ = os.path.join(HERE, "_build")
NVCC = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-lineinfo", "-std=c++17",
         "-Xcompiler", "-fPIC", "--expt-relaxed-constexpr", "-Xptxas", "-v"]


def _sources():
    return sorted(f for f in os.listdir(CSRC) if f.endswith(".cu"))


def _deps_mtime():
    files = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if not f.endswith(".cpp")] + [os.path.join(HERE, "..", "include", "aq.h")]
    return max(os.path.getmtime(f) for f in files)


def _compile(src):
    obj = os.path.join(OBJ, src[:-3] + ".o")
    cmd = [NVCC, *FLAGS, "-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    with open(obj + ".log", "w") as f:
        f.write(" ".join(cmd) + "\n" + r.stdout + r.stderr)
    if r.returncode != 0:
        raise RuntimeError(f"nvcc failed on {src}:\n{r.stdout}\n{r.stderr}")
    return obj


def torch_key() -> str:
    """What a binary of _aq_torch.so belongs to: this interpreter and its torch."""
    import torch
    return f"torch {torch.__version__} cxx11abi {int(torch._C._GLIBCXX_USE_CXX11_ABI)} {sysconfig.get_config_var('SOABI')}"


def _compile_torch(force: bool = False):
    """_aq_torch.so, against the torch that this interpreter has (its headers and libraries, no others).  Returns what is missing for it, or None."""
    include = sysconfig.get_paths()["include"]
    try:
        import torch
    except ImportError as e:
        return str(e)
    if shutil.which("g++") is None:
        return "no g++"
    if not os.path.exists(os.path.join(include, "Python.h")):
        return f"no Python.h in {include}"
    src, key_file, key = os.path.join(CSRC, "aq_torch.cpp"), os.path.join(OBJ, "aq_torch.key"), torch_key()
    deps = max(os.path.getmtime(src), os.path.getmtime(os.path.join(HERE, "..", "include", "aq.h")))
    if not force and os.path.exists(TORCH_OUT) and os.path.getmtime(TORCH_OUT) >= deps and os.path.exists(key_file):
        with open(key_file) as f:
            if f.read() == key:
                return None
    root = os.path.dirname(torch.__file__)
    inc = [os.path.join(root, "include"), os.path.join(root, "include", "torch", "csrc", "api", "include"), include,
           os.path.join(os.path.dirname(os.path.dirname(NVCC)), "include")]
    lib = os.path.join(root, "lib")
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", f'-DAQ_BUILT_FOR="{key}"',
           *(f"-I{i}" for i in inc), src, "-o", TORCH_OUT, f"-L{lib}", "-ltorch_python", "-ltorch", "-ltorch_cpu", "-lc10", "-lc10_cuda"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"g++ failed on aq_torch.cpp:\n{r.stdout}\n{r.stderr}")
    with open(key_file, "w") as f:
        f.write(key)
    return None


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile every .cu under csrc/ for sm_100a and link libaq.so; compile aq_torch.cpp where that can be done."""
    os.makedirs(OBJ, exist_ok=True)
    with concurrent.futures.ThreadPoolExecutor(max_workers=8) as ex:
        binding = ex.submit(_compile_torch, force)
        if force or not os.path.exists(OUT) or os.path.getmtime(OUT) < _deps_mtime():
            objs = list(ex.map(_compile, _sources()))
            cmd = [NVCC, "-shared", "-o", OUT, *objs, "-cudart", "static"]
            r = subprocess.run(cmd, capture_output=True, text=True)
            if r.returncode != 0:
                raise RuntimeError(f"link failed:\n{r.stdout}\n{r.stderr}")
            if verbose:
                print("built", OUT)
        missing = binding.result()   # (the library is there by now, whatever comes of this)
    if missing:
        print(f"{TORCH_OUT} is not built: {missing}; aq_kv8_plan, aq_kv8_append, aq_kv8_attn and aq_rope_rows cannot be called from Python", file=sys.stderr)
    return OUT


if __name__ == "__main__":
    build(force="--force" in sys.argv, verbose=True)
