"""Compile libtrdq.so (HIP kernels + C ABI) for gfx950 with hipcc, in-tree."""
import os
import shutil
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(os.path.dirname(HERE), "include")
OBJ_DIR = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libtrdq.so")
CALLS = os.path.join(HERE, "_trdq_calls.so")         # Python module: tensors -> the entry points around a block's linears

SOURCES = ["api.cpp", "rotate_quant.hip", "rotate_quant_rpr.hip", "calibrate.hip", "greedy_rotation.hip", "rotate_quant_dense.hip", "attention_share.hip", "prepare_weights.hip", "qgemm.hip", "qgemm_dma.hip", "qgemm_wide.hip", "qgemm_tiled.hip", "qgemm_direct.hip", "fused.hip", "peaks.hip",
           "api_blocks.cpp", "block_norm.hip", "fp8_quant.hip", "fp8_gemm.hip"]

# packed-FP32 instructions are switched off for every device compile
FLAGS = ["-O3", "-std=c++17", "-fPIC", "--offload-arch=gfx950", "-x", "hip",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-Wall", "-Wno-unused-function", "-Wno-inline-asm", "-I", CSRC, "-I", INCLUDE]


# per-source extra flags: keep the matrix-instruction accumulators of the pipelined product kernel
# in ordinary VGPRs (no accumulator-register copies around the loop)
SOURCE_FLAGS = {"qgemm_dma.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form"],
                "qgemm_direct.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form"],
                "qgemm_tiled.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form"],
                # ... and have the first kernel arguments delivered in registers at wave launch instead
                # of fetched by the kernel's first instructions (a fraction of a microsecond per launch)
                "rotate_quant.hip": ["-mllvm", "-amdgpu-kernarg-preload-count=16"],
                "fused.hip": ["-mllvm", "-amdgpu-kernarg-preload-count=16"],
                "fp8_gemm.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form"],
                "calibrate.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form"]}


def _compile(src, extra, obj_dir):
    obj = os.path.join(obj_dir, os.path.splitext(src)[0] + ".o")
    cmd = ["hipcc", *FLAGS, *SOURCE_FLAGS.get(src, []), *extra, "-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    out = "\n".join(l for l in (r.stdout + r.stderr).splitlines()
                    if "packed-fp32-ops" not in l and l.strip())
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed on {src}:\n{out}")
    return obj, out


def _calls_headers():
    """Where the headers of torch and Python lie."""
    import sysconfig

    from torch.utils import cpp_extension
    return [*cpp_extension.include_paths("cuda"), sysconfig.get_paths()["include"]]


def _calls_lack():
    """What block_calls.cpp needs beside its source and is not here, or None."""
    if shutil.which("g++") is None:
        return "g++"
    try:
        dirs = _calls_headers()
    except ImportError as e:
        return str(e)
    return next((h for h in ("Python.h", "torch/csrc/autograd/python_variable.h", "c10/hip/HIPStream.h")
                 if not any(os.path.exists(os.path.join(d, h)) for d in dirs)), None)


def build_calls(out=CALLS):
    """The Python module block_calls.cpp: host code only, linked to libtrdq.so beside it and to the installed torch.  Where its compiler or
    headers are missing, none is built (the C library and the rest of the binding need neither): says so, and returns None.  The
    calls that need it raise then; a module of an earlier build is never left behind."""
    if os.path.exists(out):
        os.remove(out)
    lack = _calls_lack()
    if lack:
        print(f"{os.path.basename(out)} is not built, its calls will raise: {lack} is missing", file=sys.stderr)
        return None
    import torch
    inc = [f"-isystem{p}" for p in _calls_headers()]
    libs = os.path.join(os.path.dirname(torch.__file__), "lib")
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-D__HIP_PLATFORM_AMD__=1", "-DUSE_ROCM=1",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch.compiled_with_cxx11_abi())}", "-I", INCLUDE, *inc, os.path.join(CSRC, "block_calls.cpp"), "-o", out,
           "-L", HERE, "-ltrdq", "-Wl,-rpath,$ORIGIN", "-L", libs, "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_hip", f"-Wl,-rpath,{libs}"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("g++ failed on block_calls.cpp:\n" + r.stderr)
    return out


def build(verbose=False, extra=(), lib=None, obj_dir=None):
    """Compiles every source and links the library; lib / obj_dir name another output (a build with
    extra preprocessor switches, e.g. the phase probe) beside the default one."""
    lib = lib or LIB
    obj_dir = obj_dir or OBJ_DIR
    os.makedirs(obj_dir, exist_ok=True)
    with ThreadPoolExecutor(max_workers=min(8, len(SOURCES))) as ex:
        results = list(ex.map(lambda s: _compile(s, list(extra), obj_dir), SOURCES))
    if verbose:
        for _, out in results:
            if out:
                print(out)
    objs = [o for o, _ in results]
    cmd = ["hipcc", "-shared", "-fPIC", "--offload-arch=gfx950", "-Wl,-soname,libtrdq.so", "-o", lib, *objs]
    subprocess.run(cmd, check=True)
    if lib == LIB:
        build_calls()
    return lib


if __name__ == "__main__":
    print(build(verbose=True, extra=sys.argv[1:]))
