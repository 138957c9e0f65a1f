"""Build libquartz.so in-tree with hipcc for gfx950, and the compiled half of the decoding
helpers (_decoding.so, host code on torch's C++ API) with g++.

Every HIP source is compiled with fp contraction off (the quantizer's
products must round to fp32 before the half-even rounding) and without
packed-fp32 instructions; fp32 division stays IEEE (hipcc's default).
"""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libquartz.so")
BINDING = os.path.join(HERE, "_decoding.so")
BINDING_SOURCE = "decoding_binding.cpp"
SOURCES = ["abi.hip", "quantize_lzs.hip", "pack_weight.hip", "w4a4_gemm.hip", "w4a4_linear.hip",
           "w4a4_gemm_plain.hip", "w4a4_linear_asym.hip", "w4a4_wide.hip", "w4a4_wide_modes.hip",
           "w4a4_wide_conv.hip", "w4a4_gemm_conv.hip", "scratch.hip",
           "attention.hip", "attention_fused.hip", "abi_decoding.hip", "mxfp4_quantize.hip",
           "mxfp4_linear.hip", "rotary.hip", "paged_attention.hip", "prompt_attention.hip",
           "paged_keep.hip"]

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared",
    "-ffp-contract=off", "-fno-fast-math",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-command-line-argument",
]


def hipcc() -> str:
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    return os.path.join(rocm, "bin", "hipcc")


def binding_flags() -> tuple[list, list]:
    """g++ flags (compile, link) of the binding: the installed torch's headers and libraries."""
    import sysconfig

    import torch
    base = os.path.dirname(torch.__file__)
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    compile_flags = ["-O2", "-std=c++17", "-fPIC", "-D__HIP_PLATFORM_AMD__", "-DUSE_ROCM",
                     f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
                     "-isystem", os.path.join(base, "include"),
                     "-isystem", os.path.join(base, "include", "torch", "csrc", "api", "include"),
                     "-isystem", os.path.join(rocm, "include"),
                     "-isystem", sysconfig.get_paths()["include"], "-Wall"]
    link_flags = ["-L", os.path.join(base, "lib"), "-lc10", "-lc10_hip", "-ltorch_cpu", "-ltorch_python",
                  "-L", HERE, "-lquartz", "-Wl,-rpath,$ORIGIN"]
    return compile_flags, link_flags


def _compile(command: list, src: str, folder: str, verbose: bool) -> tuple:
    """Compile one source of csrc into `folder`: (source, object, whether it failed, messages)."""
    noise = "is not a recognized feature for this target"
    obj = os.path.join(folder, os.path.splitext(src)[0] + ".o")
    cmd = [*command, "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-c", "-o", obj, os.path.join(CSRC, src)]
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, capture_output=True, text=True)
    err = "\n".join(l for l in res.stderr.splitlines() if noise not in l)
    return src, obj, res.returncode != 0, err


def _objects(results: list, target: str, verbose: bool) -> list:
    failed = [r[0] for r in results if r[2]]
    for src, _, _, err in results:
        if err.strip() and (verbose or failed):
            sys.stderr.write(f"{src}:\n{err}\n")
    if failed:
        raise RuntimeError(f"compiling {os.path.basename(target)} failed: " + ", ".join(failed))
    return [r[1] for r in results]


def _link(target: str, command: list) -> None:
    tmp = target + ".tmp"
    res = subprocess.run([*command, "-o", tmp], capture_output=True, text=True)
    if res.returncode != 0:
        sys.stderr.write(res.stderr + "\n")
        raise RuntimeError(f"linking {os.path.basename(target)} failed")
    os.replace(tmp, target)


def build(verbose: bool = False) -> str:
    """Compile every source to an object in parallel (each GEMM output mode is
    its own translation unit), then link libquartz.so, which needs hipcc alone, and
    after it the binding, which needs torch, Python's headers and g++ too."""
    import concurrent.futures
    import tempfile

    compile_flags = [f for f in HIPCC_FLAGS if f != "-shared"]
    workers = max(1, min(len(SOURCES) + 1, os.cpu_count() or 1))
    with tempfile.TemporaryDirectory(prefix="quartz_build_") as tmpdir, \
            concurrent.futures.ThreadPoolExecutor(max_workers=workers) as ex:
        binding = ex.submit(lambda: _compile(["g++", *binding_flags()[0]], BINDING_SOURCE, tmpdir, verbose))
        results = list(ex.map(lambda src: _compile([hipcc(), *compile_flags], src, tmpdir, verbose), SOURCES))
        _link(LIB, [hipcc(), "--offload-arch=gfx950", "-shared", "-fPIC", *_objects(results, LIB, verbose)])
        _link(BINDING, ["g++", "-shared", "-fPIC", *_objects([binding.result()], BINDING, verbose),
                        *binding_flags()[1]])
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
