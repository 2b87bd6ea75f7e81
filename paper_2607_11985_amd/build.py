"""Build libvqc.so in-tree with hipcc for gfx950 (no JIT, no caches elsewhere), and the layers'
torch extension where torch is installed (the C library needs neither torch nor Python).

    python -m paper_2607_11985_amd.build
"""
from __future__ import annotations

import importlib.util
import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
BUILD = os.path.join(PKG, "_build")
LIB = os.path.join(BUILD, "libvqc.so")
SOURCES = ["api.cpp", "planner.cpp", "qasm.cpp", "jit.cpp", "jit_compile.cpp", "kernels.hip",
           "layers_api.cpp", "layer_norm.hip", "linear.hip",
           "linear_quantized.hip", "log_probs.hip", "verify.hip"]
HELPER = os.path.join(BUILD, "vqc_jitc")  # compiles one generated kernel per process
PROBES = os.path.join(BUILD, "libvqc_probes.so")  # peak microbenchmarks (bench.py --probe)
TORCH_EXT = os.path.join(BUILD, "vqc_torch.so")  # the layers on torch tensors (layers.py)
# headers compiled again at run time for each circuit's kernels (embedded as text)
JIT_HEADERS = [("vqc_structs.h", os.path.join(CSRC, "vqc_structs.h")),
               ("vqc_device.h", os.path.join(CSRC, "vqc_device.h"))]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
CXX = os.environ.get("CXX", "g++")  # host code only

# Packed-FP32 instructions are disabled for every device compilation.
# SimplifyCFG must not sink / hoist the near-identical cases of the register-
# position switches into one block: the merged block selects between the
# amplitude variables through pointers, which pins the whole register tile in
# scratch memory.
DEVICE_FLAGS = ["--offload-arch=gfx950", "-Xclang", "-target-feature", "-Xclang",
                "-packed-fp32-ops", "-mllvm", "-simplifycfg-sink-common=false",
                "-mllvm", "-simplifycfg-hoist-common=false"]
COMMON = ["-O3", "-std=c++17", "-fPIC", "-Wall", "-I", INCLUDE, "-I", CSRC]


def _run(cmd, verbose):
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.check_call(cmd)


def write_embedded_headers() -> str:
    """C++ source holding the run-time compiler's headers as string literals."""
    out = os.path.join(BUILD, "jit_headers.cpp")
    parts = ["// generated by build.py from the shared headers; do not edit",
             "namespace vqc {", f"extern const int kJitHeaderCount = {len(JIT_HEADERS)};",
             "extern const char* const kJitHeaderNames[] = {" +
             ", ".join(f'"{n}"' for n, _ in JIT_HEADERS) + "};",
             "extern const char* const kJitHeaderSources[] = {"]
    for _, path in JIT_HEADERS:
        text = open(path).read()
        assert ")VQCSRC\"" not in text
        parts.append('R"VQCSRC(' + text + ')VQCSRC",')
    parts += ["};", "}  // namespace vqc", ""]
    text = "\n".join(parts)
    if os.path.exists(out):
        with open(out) as f:
            if f.read() == text:
                return out
    # written whole and renamed into place: a compiler in another process may
    # be reading the old file
    tmp = f"{out}.{os.getpid()}.tmp"
    with open(tmp, "w") as f:
        f.write(text)
    os.replace(tmp, out)
    return out


def torch_ext_flags():
    """Compiler and linker flags of an extension of the installed torch (no GPU code in it)."""
    import sysconfig

    import torch
    root = os.path.dirname(torch.__file__)
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    compile_flags = ["-O2", "-std=c++17", "-fPIC", "-Wall", "-D__HIP_PLATFORM_AMD__=1",
                     "-DUSE_ROCM=1", "-DTORCH_EXTENSION_NAME=vqc_torch",
                     f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}"]
    for inc in (os.path.join(root, "include"),
                os.path.join(root, "include", "torch", "csrc", "api", "include"),
                sysconfig.get_paths()["include"], os.path.join(rocm, "include")):
        compile_flags += ["-isystem", inc]
    link_flags = ["-L" + os.path.join(root, "lib")] + \
        ["-l" + lib for lib in ("c10", "torch", "torch_cpu", "torch_hip", "c10_hip",
                                "torch_python")]
    return compile_flags, link_flags


def _run_all(cmds, verbose):
    """Runs independent compile commands concurrently; fails on the first error."""
    procs = []
    for cmd in cmds:
        if verbose:
            print(" ".join(cmd), flush=True)
        procs.append((cmd, subprocess.Popen(cmd)))
    bad = [cmd for cmd, p in procs if p.wait() != 0]
    if bad:
        raise subprocess.CalledProcessError(1, bad[0])


def build_library(verbose: bool = False) -> str:
    """Compile every source, link libvqc.so and the vqc_jitc helper; always rebuilds."""
    os.makedirs(BUILD, exist_ok=True)
    emb = write_embedded_headers()
    emb_obj = os.path.join(BUILD, "jit_headers.o")
    cmds = [[HIPCC] + COMMON + ["-c", emb, "-o", emb_obj]]
    objs = [emb_obj]
    for src in SOURCES:
        path = os.path.join(CSRC, src)
        obj = os.path.join(BUILD, os.path.splitext(src)[0] + ".o")
        lang = ["-x", "hip"] if src.endswith(".hip") else []
        cmds.append([HIPCC] + COMMON + DEVICE_FLAGS + lang + ["-c", path, "-o", obj])
        objs.append(obj)
    main_obj = os.path.join(BUILD, "jitc_main.o")
    cmds.append([HIPCC] + COMMON + ["-c", os.path.join(CSRC, "jitc_main.cpp"), "-o", main_obj])
    probes_tmp = PROBES + ".tmp"
    cmds.append([HIPCC] + COMMON + DEVICE_FLAGS + ["-shared", "-x", "hip",
                                                   os.path.join(CSRC, "probes.hip"), "-o",
                                                   probes_tmp])
    _run_all(cmds, verbose)
    os.replace(probes_tmp, PROBES)
    tmp = LIB + ".tmp"
    _run([HIPCC, "-shared", "-fPIC"] + DEVICE_FLAGS + objs + ["-o", tmp, "-lhiprtc"], verbose)
    os.replace(tmp, LIB)
    tmp = HELPER + ".tmp"
    helper_objs = [main_obj, os.path.join(BUILD, "jit_compile.o"), emb_obj]
    _run([HIPCC] + helper_objs + ["-o", tmp, "-lhiprtc"], verbose)
    os.replace(tmp, HELPER)
    return LIB


def build_all(verbose: bool = False, torch_extension: bool = True) -> list:
    """libvqc.so and, unless told otherwise, the torch extension that links to it."""
    if not torch_extension:
        return [build_library(verbose)]
    os.makedirs(BUILD, exist_ok=True)
    compile_flags, link_flags = torch_ext_flags()
    obj = os.path.join(BUILD, "torch_layers.o")
    with ThreadPoolExecutor(1) as pool:  # beside the library's sources
        compiled = pool.submit(_run, [CXX] + compile_flags + [
            "-I", INCLUDE, "-c", os.path.join(CSRC, "torch_layers.cpp"), "-o", obj], verbose)
        build_library(verbose)
        compiled.result()
    # the library is found next to it at run time; the same file as the ctypes binding loads
    tmp = TORCH_EXT + ".tmp"
    _run([CXX, "-shared", obj, "-o", tmp, "-L" + BUILD, "-l:libvqc.so"] + link_flags +
         ["-Wl,-rpath,$ORIGIN"], verbose)
    os.replace(tmp, TORCH_EXT)
    return [LIB, TORCH_EXT]


if __name__ == "__main__":
    have_torch = importlib.util.find_spec("torch") is not None
    if not have_torch:
        print("torch is not installed: the layers' torch extension is not built", file=sys.stderr)
    print("\n".join(build_all("-q" not in sys.argv, have_torch)))
