"""Builds libnp.so (the C-ABI CUDA library) in-tree with nvcc for sm_100a, and the compiled part of the Python binding."""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
import sysconfig
import warnings
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(ROOT, "include")
OBJ_DIR = os.path.join(HERE, "build")
LIB_PATH = os.path.join(HERE, "libnp.so")
BIND_SOURCE = os.path.join(CSRC, "np_attn_bind.cpp")
BIND_PATH = os.path.join(HERE, "np_attn_bind.so")

SOURCES = ["np_api.cu", "np_predict.cu", "np_topk.cu", "np_centroid.cu", "np_delta.cu", "np_scatter.cu", "np_mlp.cu", "np_mlp_tc.cu", "np_mlp_chain_alu.cu", "np_mlp_slices.cu", "np_mlp_rows.cu", "np_mlp_batch.cu", "np_mlp_dense.cu", "np_static.cu", "np_io.cu", "np_trunk.cu", "np_predict_tc.cu", "np_kv.cu", "np_attn_decode.cu", "np_attn_prompt.cu", "np_kv_rows.cu", "np_attn_shared.cu", "np_attn_rest.cu"]

NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "--use_fast_math", "-Xcompiler", "-fPIC,-O2,-Wall,-Wno-unused-function",
]


def _nvcc() -> str:
    nvcc = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(nvcc):
        raise RuntimeError("nvcc not found; the CUDA library cannot be built")
    return nvcc


def _stale(target: str, deps) -> bool:
    if not os.path.exists(target):
        return True
    t = os.path.getmtime(target)
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = False, verbose: bool = False, ptxas_info: bool = False) -> str:
    """Compile every kernel file and link ``libnp.so``; returns its path."""
    nvcc = _nvcc()
    os.makedirs(OBJ_DIR, exist_ok=True)
    headers = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".h", ".cuh"))]
    headers.append(os.path.join(INCLUDE, "np.h"))
    headers.append(os.path.abspath(__file__))
    jobs = []
    objs = []
    for src in SOURCES:
        s = os.path.join(CSRC, src)
        o = os.path.join(OBJ_DIR, src.replace(".cu", ".o"))
        objs.append(o)
        if force or ptxas_info or _stale(o, [s] + headers):
            cmd = [nvcc, *NVCC_FLAGS, "-I", INCLUDE, "-I", CSRC, "-c", s, "-o", o]
            if ptxas_info:
                cmd[1:1] = ["-Xptxas", "-v"]
            jobs.append(cmd)

    def run(cmd):
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError("nvcc failed:\n" + " ".join(cmd) + "\n" + r.stdout + r.stderr)
        return r.stdout + r.stderr

    with ThreadPoolExecutor(max_workers=min(8, max(1, len(jobs)))) as ex:
        for out in ex.map(run, jobs):
            if (verbose or ptxas_info) and out.strip():
                print(out)
    if jobs or force or _stale(LIB_PATH, objs):
        run([nvcc, "-shared", "-o", LIB_PATH, *objs, "-cudart", "static", "-lpthread"])
    _build_binding(nvcc, force)
    return LIB_PATH


def bind_target() -> str:
    """What a compiled binding is good for: this torch and this interpreter."""
    import torch

    return f"torch {torch.__version__}, python {sys.version}"


def _build_binding(nvcc: str, force: bool) -> None:
    """``np_attn_bind.so``: a CPython module over libnp.so and torch's tensors.  Built again when torch or the interpreter changes.  Where it
    cannot be built (no torch, no headers of torch's or the interpreter's, no g++) there is none afterwards, and the calls that need it
    say so; the library does not need it."""
    made_by = os.path.join(OBJ_DIR, "np_attn_bind.made_by")
    try:
        import torch

        how = bind_target()
        same = os.path.exists(made_by) and open(made_by).read() == how
        if not force and same and not _stale(BIND_PATH, [BIND_SOURCE, os.path.join(INCLUDE, "np.h"), os.path.abspath(__file__)]):
            return
        home = os.path.dirname(os.path.abspath(torch.__file__))
        cuda = os.path.dirname(os.path.dirname(os.path.realpath(nvcc)))
        cmd = ["g++", "-O2", "-fPIC", "-shared", "-std=c++17", "-Wall", "-Wno-unknown-pragmas", "-I", INCLUDE, "-I", sysconfig.get_paths()["include"]]
        for d in (os.path.join(home, "include"), os.path.join(home, "include", "torch", "csrc", "api", "include"), os.path.join(cuda, "include")):
            cmd += ["-isystem", d]
        cmd += [f'-DNP_BUILT_FOR="{how}"', BIND_SOURCE, "-o", BIND_PATH, "-L", os.path.join(home, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_cuda",
                "-L", HERE, "-lnp", "-Wl,-rpath,$ORIGIN"]
        r = subprocess.run(cmd, capture_output=True, text=True)
        why = "" if r.returncode == 0 else "g++ failed:\n" + " ".join(cmd) + "\n" + r.stdout + r.stderr
    except (ImportError, OSError) as e:
        why = str(e)
    if why:
        if os.path.exists(BIND_PATH):
            os.remove(BIND_PATH)
        warnings.warn(f"np_attn_bind.so could not be built; the cache and attention calls of the Python binding need it: {why}")
        return
    with open(made_by, "w") as f:
        f.write(how)


if __name__ == "__main__":
    path = build(force="--force" in sys.argv, verbose=True, ptxas_info="--ptxas" in sys.argv)
    print(path)
