"""Build libgoodroute.so for gfx950 with hipcc (in-tree, next to the sources)."""
from __future__ import annotations

import os
import re
import subprocess
import sys

_HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(_HERE)
CSRC = os.path.join(_HERE, "csrc")
LIB = os.path.join(CSRC, "libgoodroute.so")
SOURCES = ["api.hip", "status.hip", "score.hip", "experts_api.hip", "experts.hip", "linear.hip", "clip.hip"]


def hipcc_command() -> list:
    return ["hipcc", "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared",
            "-ffp-contract=off",
            # packed-FP32 instructions stay off: ordinary float code must not be fused into them
            "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
            "-Rpass-analysis=kernel-resource-usage",      # (what check_spills reads)
            "-I", os.path.join(ROOT, "include"),
            "-o", LIB] + [os.path.join(CSRC, s) for s in SOURCES]


# Kernels whose sums are bound to registers behind the compiler's back: with a vector register spilled they are wrong.
NOTHING_SPILLED = ("k_linear_tiles",)


def check_spills(remarks: str) -> None:
    """Raises where the compiler's remarks say that one of those kernels spills vector registers or uses scratch memory, or say nothing of it."""
    seen = set()
    for part in remarks.split("remark: Function Name: ")[1:]:
        name = part.split()[0]
        for kernel in NOTHING_SPILLED:
            if kernel not in name:
                continue
            seen.add(kernel)
            for what in (r"VGPRs Spill", r"ScratchSize \[bytes/lane\]"):
                m = re.search(what + r": (\d+)", part)
                if m is None or int(m.group(1)):
                    raise RuntimeError(f"{name}: {m.group(0) if m else 'no word of ' + what}, and its sums are wrong if any vector register is spilled")
    if seen != set(NOTHING_SPILLED):
        raise RuntimeError(f"the compiler said nothing of {sorted(set(NOTHING_SPILLED) - seen)}")


def build_library(verbose: bool = False) -> str:
    cmd = hipcc_command()
    if verbose:
        print(" ".join(cmd), flush=True)
    made = subprocess.run(cmd, stderr=subprocess.PIPE, text=True)
    # (a remark is a line, the line of source it names, and a mark under that)
    said = re.sub(r"^.*: remark: .*\[-Rpass-analysis=kernel-resource-usage\]\n(?:^ *\d* \|.*\n)*", "", made.stderr, flags=re.M)
    sys.stderr.write(said)
    made.check_returncode()
    try:
        check_spills(made.stderr)
    except RuntimeError:
        os.remove(LIB)
        raise
    return LIB


MARSHAL = os.path.join(CSRC, "goodroute_marshal.so")


def build_marshal(verbose: bool = False) -> str:
    """The binding's argument marshalling (host code only, against torch's headers)."""
    import sysconfig

    import torch
    at = os.path.dirname(torch.__file__)
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
           "-D__HIP_PLATFORM_AMD__=1", "-I", sysconfig.get_path("include"), "-I", os.path.join(at, "include"),
           "-I", os.path.join(at, "include", "torch", "csrc", "api", "include"), "-I", "/opt/rocm/include",
           "-o", MARSHAL, os.path.join(CSRC, "marshal.cpp"), "-L", os.path.join(at, "lib"), "-ltorch_python", "-lc10_hip"]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.run(cmd, check=True)
    return MARSHAL


PROBE = os.path.join(CSRC, "probe_valu_issue")


def build_probe(verbose: bool = False) -> str:
    """The stand-alone microbenchmark behind the vector-ALU issue model (not part of the library)."""
    cmd = ["hipcc", "--offload-arch=gfx950", "-O3", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
           "-o", PROBE, PROBE + ".hip"]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.run(cmd, check=True)
    return PROBE


if __name__ == "__main__":
    build_library(verbose=True)
    build_marshal(verbose=True)
    build_probe(verbose=True)
