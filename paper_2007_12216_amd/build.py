"""Build the HIP library in-tree: paper_2007_12216_amd/librnswino.so (gfx950), and _decoder.so, the extension module of decoder.py."""
from __future__ import annotations

import importlib.util
import os
import subprocess
import tempfile

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "librnswino.so")
SOURCES = ("rnswino.hip", "plan_math.cpp")
DECODER = "decoder.hip"  # the decoder operators: an object of its own, compiled beside the others
EXTENSION = os.path.join(PKG, "_decoder.so")  # their calls from Python (decoder.py)


def compile_command(out: str) -> list:
    """The hipcc command that compiles every source for gfx950 and links them to `out`."""
    cmd = ["hipcc", "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared",
           "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
           # matrix-core results straight into ordinary vector registers: no accumulator-register copies in the
           # epilogues, and fewer registers per wave
           "-mllvm", "-amdgpu-mfma-vgpr-form=1",
           "-Wno-unused-command-line-argument",
           "-I", os.path.join(ROOT, "include"), "-I", CSRC]
    cmd += [os.path.join(CSRC, s) for s in SOURCES]
    return cmd + ["-o", out]


def object_command(source: str, out: str) -> list:
    """The hipcc command that compiles one source of csrc/, with the same flags, to the object file `out`."""
    shared = [a for a in compile_command(out) if a != "-shared" and os.path.basename(a) not in SOURCES]
    return shared + ["-c", os.path.join(CSRC, source)]


def extension_command(out: str) -> list:
    """The command that compiles the extension module decoder.py calls, against the library built before it and this interpreter's torch."""
    import sysconfig
    import torch
    home = os.path.dirname(torch.__file__)
    includes = [os.path.join(home, "include"), os.path.join(home, "include", "torch", "csrc", "api", "include"), os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "include"),
                sysconfig.get_paths()["include"], os.path.join(ROOT, "include")]
    return ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-D__HIP_PLATFORM_AMD__", "-DUSE_ROCM", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch.compiled_with_cxx11_abi())}",
            *(f"-I{d}" for d in includes), os.path.join(CSRC, "decoder_binding.cpp"), "-o", out,
            "-L" + os.path.join(home, "lib"), "-ltorch_python", "-ltorch", "-ltorch_cpu", "-ltorch_hip", "-lc10", "-lc10_hip", "-L" + PKG, "-l:" + os.path.basename(LIB), "-Wl,-rpath,$ORIGIN"]


def run_all(commands: list, verbose: bool) -> str:
    """Runs commands beside each other; their output, or an error with it."""
    if verbose:
        for cmd in commands:
            print(" ".join(cmd), flush=True)
    running = [subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True) for cmd in commands]
    printed = "\n".join(p.communicate()[0] for p in running)
    # the host pass warns that it does not know the packed-fp32 feature; that is expected
    out = "\n".join(l for l in printed.splitlines() if "packed-fp32-ops" not in l)
    failed = [cmd[0] for cmd, p in zip(commands, running) if p.returncode]
    if failed:
        raise RuntimeError(f"{failed[0]} failed:\n" + out)
    return out


def build_library(verbose: bool = False) -> str:
    """Compile every source with hipcc for gfx950, one process each, and link the shared library; with torch there, the extension module too (decoder.py, which calls it, needs torch itself)."""
    with tempfile.TemporaryDirectory() as folder:
        sources = SOURCES + (DECODER,)
        objects = [os.path.join(folder, s + ".o") for s in sources]
        out = run_all([object_command(s, o) for s, o in zip(sources, objects)], verbose)
        out += run_all([["hipcc", "--offload-arch=gfx950", "-shared", *objects, "-o", LIB]], verbose)
    if importlib.util.find_spec("torch") is not None:
        out += run_all([extension_command(EXTENSION)], verbose)
    if verbose and out.strip():
        print(out)
    return LIB


if __name__ == "__main__":
    print(build_library(verbose=True))
