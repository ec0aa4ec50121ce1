"""Builds the CUDA libraries in-tree for sm_100a with nvcc:

  libsae.so        -- the C-ABI library declared in include/sae.h
  libsae_synth.so  -- the seeded synthetic-gradient generator used by tests and the benchmark
  _host.so         -- the Python side of gradient sets and group norm (argument checks, allocation), C++ against torch;
                      left out where torch is not installed

Usage: python -m paper_2008_05823_b200.build [--force] [--verbose]
"""
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(os.path.dirname(HERE), "include")

NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17", "-fmad=false",
              "-Xcompiler", "-fPIC", "-shared"]

TARGETS = {
    "libsae.so": (["sae.cu", "sae_noalloc.cu", "sae_grads.cu", "sae_group_norm.cu"], ["sae_vec.cuh", "sae_gn_common.cuh", "sae_gn_unit.cuh", "sae_gn_stream.cuh", "sae_kernels.cuh", "sae_worker_tma.cuh", "sae_worker_fused.cuh", "sae_worker_small.cuh", "sae_topk.cuh", "sae_shard_topk.cuh", "sae_device.cuh", os.path.join(INCLUDE, "sae.h")]),
    "libsae_synth.so": (["synth_gen.cu"], []),
    "_host.so": (["host_torch.cpp"], [os.path.join(INCLUDE, "sae.h")]),
}


def _host_command(out, sources):
    """g++ against the installed torch's headers; libsae.so is found beside the module."""
    import sysconfig
    from torch.utils import cpp_extension
    cuda = os.environ.get("CUDA_HOME", "/usr/local/cuda")
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden", "-DTORCH_EXTENSION_NAME=_host"]
    for inc in cpp_extension.include_paths() + [os.path.join(cuda, "include"), sysconfig.get_paths()["include"]]:
        cmd += ["-isystem", inc]
    cmd += ["-o", out] + sources + ["-L" + HERE, "-l:libsae.so", "-Wl,-rpath,$ORIGIN"]
    for lib in cpp_extension.library_paths() + [os.path.join(cuda, "lib64")]:
        cmd.append("-L" + lib)
    return cmd + ["-lc10", "-lc10_cuda", "-ltorch_cpu", "-ltorch_cuda", "-ltorch", "-ltorch_python", "-lcudart"]


def _stale(out, deps):
    if not os.path.exists(out):
        return True
    t = os.path.getmtime(out)
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = False, verbose: bool = False):
    nvcc = os.environ.get("NVCC", "nvcc")
    outs = []
    for name, (srcs, hdrs) in TARGETS.items():
        out = os.path.join(HERE, name)
        src_paths = [os.path.join(CSRC, s) for s in srcs]
        dep_paths = src_paths + [h if os.path.isabs(h) else os.path.join(CSRC, h) for h in hdrs]
        if force or _stale(out, dep_paths):
            extra = os.environ.get("SAE_NVCC_EXTRA", "").split()
            if src_paths[0].endswith(".cpp"):
                try:
                    cmd = _host_command(out, src_paths)
                except ImportError:
                    print(f"{name} is not built: torch is not installed", file=sys.stderr)
                    continue
                subprocess.check_call(cmd)
                outs.append(out)
                continue
            cmd = [nvcc] + NVCC_FLAGS + extra + (["-Xptxas", "-v"] if verbose else []) + ["-o", out] + src_paths
            subprocess.check_call(cmd)
        outs.append(out)
    return outs


if __name__ == "__main__":
    for o in build(force="--force" in sys.argv, verbose="--verbose" in sys.argv):
        print(o)
