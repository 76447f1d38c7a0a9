"""Builds libsparseconv.so (HIP kernels + C ABI) in-tree for gfx950, and the Python side of the text model's operators."""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libsparseconv.so")
TORCH_LIB = os.path.join(HERE, "_text_torch.so")
SOURCES = ["kernels.hip", "matrix_f32.hip", "matrix_f16.hip", "probes.hip", "api.cpp", "plan.cpp", "matrix_plan.cpp", "host_csr.cpp",
           "embed.hip", "int8.hip", "text_api.cpp"]

# packed fp32 VALU forms are switched off for the device pass (the host pass
# prints a harmless "not a recognized feature" note for the same flag)
HIPCC_FLAGS = [
    "-O3", "-std=c++17", "--offload-arch=gfx950", "-fPIC",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-command-line-argument",
]


def build(verbose: bool = False) -> str:
    """Compiles every source (side by side) and links them.  The Python side of the text model's operators is built as well where PyTorch
    is there; the library needs neither it nor its compiler."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    with tempfile.TemporaryDirectory() as objects:
        cmds = [[hipcc] + HIPCC_FLAGS + ["-c", "-o", os.path.join(objects, s + ".o"), os.path.join(CSRC, s)] for s in SOURCES]
        torch_lib = os.path.join(objects, os.path.basename(TORCH_LIB))
        torch_side = torch_command(torch_lib)
        if torch_side is None and verbose:
            print("PyTorch is not there: the library without " + os.path.basename(TORCH_LIB), flush=True)
        link = [hipcc] + HIPCC_FLAGS + ["-shared", "-o", LIB] + [c[-2] for c in cmds]
        running = [(c, subprocess.Popen(c, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)) for c in cmds + ([torch_side] if torch_side else [])]
        done = [(c, p.communicate()[0], p.returncode) for c, p in running]
        if all(rc == 0 for _, _, rc in done[:len(cmds)]):
            res = subprocess.run(link, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
            done.insert(len(cmds), (link, res.stdout, res.returncode))
        if torch_side and done[-1][2] == 0:      # moved into place whole: another process may be about to load it
            shutil.copyfile(torch_lib, TORCH_LIB + ".new")
            os.replace(TORCH_LIB + ".new", TORCH_LIB)
    for cmd, text, rc in done:
        if verbose:
            print(" ".join(cmd), flush=True)
        out = "\n".join(l for l in text.splitlines() if "packed-fp32-ops" not in l)
        if rc != 0:
            raise RuntimeError(os.path.basename(cmd[0]) + " failed:\n" + out)
        if verbose and out.strip():
            print(out)
    return LIB


def torch_command(path: str):
    """The compiler's call that makes `path`, the Python side of the text model's operators (checks and allocation on PyTorch tensors, host
    code), or None where PyTorch is not there."""
    try:
        import torch
        from torch.utils import cpp_extension
    except ImportError:
        return None
    import sysconfig
    lib = os.path.join(os.path.dirname(torch.__file__), "lib")
    return ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
            f"-I{sysconfig.get_paths()['include']}", *[f"-I{p}" for p in cpp_extension.include_paths()],
            "-o", path, os.path.join(CSRC, "text_torch.cpp"), f"-L{lib}", f"-Wl,-rpath,{lib}", "-ltorch_python", "-ltorch_cpu", "-lc10"]


_SANITIZE = ["-fsanitize=address,undefined", "-fno-sanitize-recover=undefined", "-fno-omit-frame-pointer", "-g", "-O1"]


def _build_dir() -> str:
    path = os.path.join(os.path.dirname(HERE), "_build")
    os.makedirs(path, exist_ok=True)
    return path


def _sanitized(driver: str, exe: str, sources, objects=()) -> list:
    """The compiler's call for a sanitizer driver of tests/sanitize, linked with host sources of the library."""
    return ["g++", "-std=c++17", *_SANITIZE, "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-o", exe,
            os.path.join(os.path.dirname(HERE), "tests", "sanitize", driver), *objects, *[os.path.join(CSRC, f) for f in sources],
            "-L/opt/rocm/lib", "-Wl,-rpath,/opt/rocm/lib", "-lamdhip64", "-lm"]


def _run_all(cmds, verbose: bool) -> None:
    for cmd in cmds:
        if verbose:
            print(" ".join(cmd), flush=True)
        res = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
        if res.returncode != 0:
            raise RuntimeError("sanitizer build failed:\n" + res.stdout)


def build_sanitize(verbose: bool = False) -> str:
    """Host-only build for the sanitizer check: CSR encoder, planner and the C ABI (no kernels; the launch
    functions are stand-ins that report "not supported"), the CPU oracle and tests/sanitize/driver.cpp in one
    executable compiled with -fsanitize=address,undefined.  Returns its path; needs no GPU."""
    exe, oracle_o = os.path.join(_build_dir(), "sanitize_driver"), os.path.join(_build_dir(), "oracle_sanitize.o")
    _run_all([["gcc", "-std=c11", "-ffp-contract=off", "-c", *_SANITIZE, "-o", oracle_o, os.path.join(os.path.dirname(HERE), "oracle", "sparse_conv_oracle.c")],
              _sanitized("driver.cpp", exe, ("api.cpp", "plan.cpp", "matrix_plan.cpp", "host_csr.cpp", "no_device.cpp"), [oracle_o])], verbose)
    return exe


def build_sanitize_text(verbose: bool = False) -> str:
    """The same for the text model's entry points (text_api.cpp) and tests/sanitize/text_driver.cpp."""
    exe = os.path.join(_build_dir(), "sanitize_text_driver")
    _run_all([_sanitized("text_driver.cpp", exe, ("text_api.cpp", "no_device.cpp"))], verbose)
    return exe


if __name__ == "__main__":
    if "--sanitize" in sys.argv[1:]:
        print(build_sanitize(verbose=True))
        print(build_sanitize_text(verbose=True))
    else:
        print(build(verbose=True))
