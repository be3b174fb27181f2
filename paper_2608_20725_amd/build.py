"""Builds libim2win.so (the C-ABI library and its gfx950 kernels) and, where torch
is installed, _seq_cache.so (the Python binding of the cache's calls) in-tree.

    python -m paper_2608_20725_amd.build [--library]     # --library: without the binding

Every HIP source is compiled for gfx950 only, with packed fp32 VALU
instructions disabled (``-packed-fp32-ops``): the fp32 path uses plain
v_fma_f32 / v_fmac_f32.
"""
from __future__ import annotations

import importlib.util
import os
import shutil
import subprocess
import sys
import sysconfig
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libim2win.so")
SOURCES = ["api.cpp", "plan.cpp", "chunked.cpp", "transform.hip", "conv_fp32.hip", "conv_fp16.hip", "conv_fp16_col.hip", "conv_fp32_dma.hip", "conv_fp16_seg.hip", "conv_fp32_mfma.hip", "conv_fp16_stem.hip", "conv_fp16_direct.hip", "conv_fp32_stem.hip", "conv_fp32_cols.hip",
           "seq_api.cpp", "seq_norm.hip", "seq_bias.hip", "seq_attn_fwd.hip", "seq_attn_decode.hip",
           "seq_attn_bwd.hip", "seq_cache_api.cpp", "seq_rotary.hip", "seq_cache.hip", "seq_paged.hip"]

# The Python binding of the small serving calls: host code against torch's headers.
BINDING = os.path.join(HERE, "_seq_cache.so")
BINDING_SOURCE = "py_cache.cpp"

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = [
    "-x", "hip", "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function",
    "-I", os.path.join(ROOT, "include"),
]


def _run(cmd):
    p = subprocess.run(cmd, capture_output=True, text=True)
    # the host pass does not know the gfx950 feature name: drop that warning
    noise = [l for l in (p.stdout + p.stderr).splitlines()
             if l.strip() and "packed-fp32-ops" not in l]
    return p.returncode, noise


def _torch_folder():
    """torch's package folder, or None."""
    spec = importlib.util.find_spec("torch")
    return list(spec.submodule_search_locations)[0] if spec and spec.submodule_search_locations else None


def _binding_commands(torch, obj, libdir, out):
    """Compile and link commands of the binding, against torch's package folder and the library in ``libdir``."""
    cxx = os.environ.get("CXX", "g++")
    rocm = os.path.dirname(os.path.dirname(os.path.realpath(HIPCC)))
    headers = [sysconfig.get_paths()["include"], os.path.join(rocm, "include"), os.path.join(torch, "include"),
               os.path.join(torch, "include", "torch", "csrc", "api", "include")]
    # HIP's and torch's headers ask which platform they are compiled for
    compile_cmd = [cxx, "-O2", "-std=c++17", "-fPIC", "-Wall", "-D__HIP_PLATFORM_AMD__=1", "-DUSE_ROCM=1",
                   "-I", os.path.join(ROOT, "include")]
    for h in headers:
        compile_cmd += ["-isystem", h]
    compile_cmd += ["-c", os.path.join(CSRC, BINDING_SOURCE), "-o", obj]
    link_cmd = [cxx, "-shared", obj, "-L", libdir, "-l:libim2win.so", "-Wl,-rpath,$ORIGIN", "-L", os.path.join(torch, "lib"),
                "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_hip", "-o", out]
    return compile_cmd, link_cmd


def _result(cmd, result, verbose, what):
    """Prints a command and what it said; a failed one raises."""
    rc, noise = result
    if verbose:
        print(" ".join(cmd), flush=True)
    if noise and (verbose or rc != 0):
        sys.stderr.write("\n".join(noise) + "\n")
    if rc != 0:
        raise RuntimeError(what)


def build(verbose: bool = False, binding: bool = True) -> str:
    """Compiles every source to an object (in parallel), then links them.

    ``binding`` False, or no torch: the library alone, without anything of torch.
    A binding of another library is not left beside it: both are replaced when
    both are linked, and where only the library is built an old binding goes."""
    from concurrent.futures import ThreadPoolExecutor
    torch = _torch_folder() if binding else None
    if binding and torch is None:
        print("torch is not installed: libim2win.so is built without _seq_cache.so", flush=True)
    objdir = os.path.join(ROOT, "_build", "obj")
    os.makedirs(objdir, exist_ok=True)
    link = tempfile.mkdtemp(prefix="link", dir=os.path.join(ROOT, "_build"))
    try:
        lib, module = os.path.join(link, os.path.basename(LIB)), os.path.join(link, os.path.basename(BINDING))
        compile_flags = [f for f in FLAGS if f != "-shared"]
        objects = [os.path.join(objdir, os.path.splitext(s)[0] + ".o") for s in SOURCES]
        jobs = [[HIPCC] + compile_flags + ["-c", os.path.join(CSRC, s), "-o", obj] for s, obj in zip(SOURCES, objects)]
        what = ["hipcc failed building libim2win.so"] * len(jobs)
        if torch:
            binding_compile, binding_link = _binding_commands(
                torch, os.path.join(objdir, os.path.splitext(BINDING_SOURCE)[0] + ".o"), link, module)
            jobs.append(binding_compile)
            what.append("compiling _seq_cache.so, the binding to torch, failed; build(binding=False) (--library) builds "
                        "libim2win.so alone")
        workers = max(1, min(len(jobs), os.cpu_count() or 1, 16))
        with ThreadPoolExecutor(workers) as ex:
            results = list(ex.map(_run, jobs))
        for cmd, result, text in zip(jobs, results, what):
            _result(cmd, result, verbose, text)
        cmd = [HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC"] + objects + ["-o", lib]
        _result(cmd, _run(cmd), verbose, "linking libim2win.so failed")
        if torch:
            _result(binding_link, _run(binding_link), verbose, "linking _seq_cache.so, the binding to torch, failed; "
                    "build(binding=False) (--library) builds libim2win.so alone")
        elif os.path.exists(BINDING):
            os.remove(BINDING)
        os.replace(lib, LIB)
        if torch:
            os.replace(module, BINDING)
    finally:
        shutil.rmtree(link, ignore_errors=True)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True, binding="--library" not in sys.argv[1:]))
