"""Builds the HIP extension in-tree, paper_2602_01469_amd/libpeagle_attn.so (gfx950 only), and the binding's compiled part,
paper_2602_01469_amd/_marshal.so (host code against the installed torch)."""
from __future__ import annotations

import os
import subprocess
import sys
import sysconfig
import warnings

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libpeagle_attn.so")
SOURCES = ["tilemap.cpp", "api.cpp", "attn_kernels.hip", "rope_kernels.hip", "cache_kernels.hip",
           "draft_scaled_kernels.hip"]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
MARSHAL = os.path.join(HERE, "_marshal.so")


def _run(cmd, what: str) -> str:
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    out = "\n".join(l for l in r.stdout.splitlines() if "not a recognized feature" not in l)
    if r.returncode != 0:
        raise RuntimeError(what + " failed:\n" + out)
    return out


def build_marshal(out: str = "", compiler: str = "g++", flags: tuple = ("-O2",)) -> str:
    import torch
    from .binding import marshal_needs
    torch_dir = os.path.dirname(torch.__file__)
    _run([compiler, *flags, "-std=c++17", "-fPIC", "-shared", "-D__HIP_PLATFORM_AMD__=1", "-DUSE_ROCM=1", f'-DPEAGLE_BUILT_FOR="{marshal_needs()}"',
          "-I" + os.path.join(torch_dir, "include"),
          "-I" + os.path.join(torch_dir, "include", "torch", "csrc", "api", "include"), "-I/opt/rocm/include",
          "-I" + sysconfig.get_paths()["include"], os.path.join(CSRC, "marshal.cpp"), "-o", out or MARSHAL, "-L" + os.path.join(torch_dir, "lib"),
          "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_hip"], compiler)
    return out or MARSHAL


def build(verbose: bool = False, sanitize_host_to: str = "") -> str:
    """Builds the library in-tree.  With `sanitize_host_to`, builds a second library at that path instead whose HOST
    code (tile-map builder, argument validation, launch drivers) carries AddressSanitizer and
    UndefinedBehaviorSanitizer; the device code is the same (no sanitizer runs on the GPU)."""
    out_path = sanitize_host_to or LIB
    opt = ["-O3", "-Xarch_host", "-O1", "-Xarch_host", "-g", "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
           "-Xarch_host", "-fno-sanitize-recover=undefined", "-Xarch_host", "-fno-omit-frame-pointer",
           "-shared-libsan"] if sanitize_host_to else ["-O3"]
    cmd = [
        HIPCC, "-x", "hip", "--offload-arch=gfx950", *opt, "-std=c++17", "-fPIC", "-shared",
        "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
        # Matrix instructions write ordinary vector registers in every kernel.  Kernels with one wave per SIMD (the
        # D=128 dK/dV kernel) would otherwise get all their accumulators in the accumulation registers and copy
        # every score out before the vector unit can touch it (that kernel: -7 %); the others are unaffected.
        "-mllvm", "-amdgpu-mfma-vgpr-form",
        "-fgpu-flush-denormals-to-zero", "-Wno-unused-command-line-argument",
        "-I", os.path.join(ROOT, "include"), "-I", CSRC,
        "-o", out_path,
    ] + [os.path.join(CSRC, s) for s in SOURCES]
    if verbose:
        cmd.insert(1, "-Rpass-analysis=kernel-resource-usage")
    out = _run(cmd, "hipcc")
    if not sanitize_host_to:
        # (the library does without: what cannot be built leaves no older one behind)
        try:
            build_marshal()
        except (RuntimeError, OSError, ImportError) as e:
            if os.path.exists(MARSHAL):
                os.remove(MARSHAL)
            warnings.warn(f"_marshal.so is not built, calls on 4-bit caches and reads will be marshalled in Python: {e}", RuntimeWarning, stacklevel=2)
    if verbose and out:
        print(out)
    return out_path


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
