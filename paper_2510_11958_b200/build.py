"""Build the CUDA library (sm_100a only) into paper_2510_11958_b200/libdmtd_b200.so, and beside it _paged.so, the argument
marshalling of the paged cache's calls.

`python -m paper_2510_11958_b200.build` or build().  nvcc cross-compiles without a GPU.
"""
import os
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
LIB = os.path.join(HERE, "libdmtd_b200.so")
BINDING = os.path.join(HERE, "_paged.so")
SOURCES = ["engine.cu", "paged.cu"]
HEADERS = ["common.cuh", "ptx.cuh", "kernels.cuh", "pass_common.cuh", "pass_stream.cuh", "pass_prologues.cuh",
           "pass_attention.cuh", "pass_attention_f32.cuh", "pass_kernel.cuh", "attention_kernel.cuh", "attention_tc05.cuh",
           "gemm_tc05.cuh", "small_pass.cuh", "host.h", "paged_common.cuh", "paged_plan.cuh", "paged_append.cuh", "paged_attention.cuh", "paged_line.cuh",
           "paged_rows.cuh", "paged_chunk.cuh"]


def _stale(made, deps) -> bool:
    if not os.path.exists(made):
        return True
    t = os.path.getmtime(made)
    deps = [os.path.join(HERE, "csrc", f) for f in deps] + [os.path.join(ROOT, "include", "dmtd.h")]
    return any(os.path.getmtime(d) > t for d in deps if os.path.exists(d))


def _made_for() -> str:
    """What the binding is compiled against besides the sources: it uses torch's C++ interface and carries no tag in its name."""
    import torch
    return f"torch {torch.__version__}, {sysconfig.get_config_var('SOABI')}"


def _binding_stale() -> bool:
    if _stale(BINDING, ["paged_binding.cpp"]):
        return True
    with open(BINDING, "rb") as f:
        return b"[made for " + _made_for().encode() + b"]" not in f.read()


def _binding_command(to):
    import torch
    from torch.utils import cpp_extension
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", "-I" + sysconfig.get_paths()["include"], "-I/usr/local/cuda/include",
           f'-DDMTD_MADE_FOR="[made for {_made_for()}]"']
    cmd += ["-isystem" + p for p in cpp_extension.include_paths()]
    cmd += [os.path.join(HERE, "csrc", "paged_binding.cpp"), "-o", to]
    for p in cpp_extension.library_paths():
        cmd += ["-L" + p, "-Wl,-rpath," + p]
    return cmd + ["-ltorch_python", "-ltorch", "-ltorch_cpu", "-lc10", "-lc10_cuda", "-L" + HERE, "-l:" + os.path.basename(LIB), "-Wl,-rpath,$ORIGIN"]


def build(force: bool = False, verbose: bool = False) -> str:
    if force or _stale(LIB, SOURCES + HEADERS):
        _build_library(verbose)
    if force or _binding_stale():
        tmp = BINDING + f".tmp{os.getpid()}"
        _run(_binding_command(tmp), verbose)
        os.replace(tmp, BINDING)
    return LIB


def _run(cmd, verbose):
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        sys.stderr.write(r.stdout + r.stderr)
        raise RuntimeError(f"{os.path.basename(cmd[0])} failed")
    if verbose:
        sys.stderr.write(r.stdout + r.stderr)


def _build_library(verbose) -> None:
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    tmp = LIB + f".tmp{os.getpid()}"
    cmd = [nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-lineinfo", "-std=c++17",
           "--use_fast_math" if False else "-DDMTD_NO_FAST_MATH", "-Xcompiler", "-fPIC", "-shared", "--threads", str(len(SOURCES)),
           "-I", os.path.join(ROOT, "include")]
    cmd += os.environ.get("DMTD_NVCC_FLAGS", "").split()      # e.g. -DDMTD_PASS_SLOTS=2 for an experiment
    if verbose:
        cmd += ["-Xptxas", "-v"]
    cmd += [os.path.join(HERE, "csrc", f) for f in SOURCES] + ["-o", tmp]
    _run(cmd, verbose)
    os.replace(tmp, LIB)


if __name__ == "__main__":
    print(build(force=True, verbose="-v" in sys.argv))
