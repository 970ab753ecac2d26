"""Build step for the HIP library: compiles csrc/*.hip for gfx950 into
_lib/libsbvr.so (in-tree, so the built library travels with the source).
``defines`` (NAME=VALUE) override launch-shape tuning macros for sweeps."""
from __future__ import annotations

import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
SOURCES = [os.path.join(HERE, "csrc", f) for f in ("api.hip", "pack.hip", "gemv_b1.hip", "gemv_b1s.hip", "gemm_sbs.hip",
                                                  "decompress.hip", "encode.hip", "prefill.hip", "api_step.hip",
                                                  "plan.hip", "cache_write.hip", "attention.hip", "norm.hip",
                                                  "logits.hip", "rotary.hip", "beam.hip", "pages.hip")]
# The encoder's binary64 arithmetic is its definition: no fused multiply-add.
SOURCE_FLAGS = {
    "encode.hip": ["-ffp-contract=off"],
    # leading scalar kernel arguments preloaded into SGPRs (batch-1 kernels)
    "gemv_b1.hip": ["-mllvm", "-amdgpu-kernarg-preload-count=8"],
    "gemv_b1s.hip": ["-mllvm", "-amdgpu-kernarg-preload-count=10"],
}
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared",
    "-Wall", "-Wno-unused-result",
    # never emit packed-fp32 VALU instructions (v_pk_{add,mul,fma}_f32)
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
]


def library_path() -> str:
    return os.path.join(HERE, "_lib", "libsbvr.so")


def probe_path() -> str:
    """The streaming-read measurement helper the benchmark loads (not part of
    the library)."""
    return os.path.join(HERE, "_lib", "libsbvr_probe.so")


def build_probe(verbose: bool = False) -> str:
    out = probe_path()
    os.makedirs(os.path.dirname(out), exist_ok=True)
    tmp = out + ".tmp%d" % os.getpid()
    cmd = [HIPCC, *FLAGS, os.path.join(HERE, "csrc", "read_probe.hip"), "-o", tmp]
    if verbose:
        print(" ".join(cmd))
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("hipcc failed:\n" + " ".join(cmd) + "\n" + r.stdout + r.stderr)
    os.replace(tmp, out)
    return out


def binding_path() -> str:
    """The extension module with the tensor helpers of the operators between
    the products (csrc/step_bind.cpp)."""
    return os.path.join(HERE, "_lib", "_sbvr_step.so")


def build_binding(verbose: bool = False) -> str | None:
    """Host code only: compiled against torch's headers, no GPU code in it.
    Where torch or the C++ compiler is missing nothing is built, and None
    returned: the library needs neither."""
    import importlib.util
    import shutil
    import sys
    import sysconfig

    out, compiler = binding_path(), os.environ.get("CXX", "g++")
    os.makedirs(os.path.dirname(out), exist_ok=True)
    missing = [name for name, there in (("torch", importlib.util.find_spec("torch")), (compiler, shutil.which(compiler)))
               if not there]
    if missing:
        if os.path.exists(out):  # made for another build of the library
            os.remove(out)
        print(f"the tensor binding is not built: {' and '.join(missing)} not found", file=sys.stderr)
        return None

    import torch
    from torch.utils.cpp_extension import include_paths, library_paths

    tmp = out + ".tmp%d" % os.getpid()
    includes = [*include_paths(), sysconfig.get_paths()["include"], os.path.join(ROOT, "include"),
                os.path.join(os.path.dirname(os.path.dirname(HIPCC)), "include")]
    cmd = [compiler, "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall", "-fvisibility=hidden",
           "-DTORCH_EXTENSION_NAME=_sbvr_step", "-DTORCH_API_INCLUDE_EXTENSION_H", "-D__HIP_PLATFORM_AMD__",
           "-D_GLIBCXX_USE_CXX11_ABI=%d" % int(torch._C._GLIBCXX_USE_CXX11_ABI),
           *(f for p in includes for f in ("-isystem", p)), os.path.join(HERE, "csrc", "step_bind.cpp"),
           *("-L" + p for p in library_paths()), "-lc10", "-ltorch_cpu", "-ltorch", "-ltorch_python", "-o", tmp]
    if verbose:
        print(" ".join(cmd))
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("g++ failed:\n" + " ".join(cmd) + "\n" + r.stdout + r.stderr)
    os.replace(tmp, out)
    return out


def build(verbose: bool = False, out: str | None = None, defines=(), jobs: int = 0) -> str:
    """Compile every source to an object (in parallel), then link libsbvr.so."""
    from concurrent.futures import ThreadPoolExecutor

    out = out or library_path()
    os.makedirs(os.path.dirname(out), exist_ok=True)
    objdir = os.path.join(os.path.dirname(out), "obj.%d" % os.getpid())
    os.makedirs(objdir, exist_ok=True)
    common = [*FLAGS, *("-D" + d for d in defines), "-I", os.path.join(ROOT, "include"),
              "-I", os.path.join(HERE, "csrc")]

    def run(cmd):
        if verbose:
            print(" ".join(cmd))
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError("hipcc failed:\n" + " ".join(cmd) + "\n" + r.stdout + r.stderr)

    objs = [os.path.join(objdir, os.path.basename(src) + ".o") for src in SOURCES]
    compile_flags = [f for f in common if f != "-shared"]
    jobs = jobs or min(len(SOURCES), os.cpu_count() or 1, 8)
    try:
        with ThreadPoolExecutor(max_workers=jobs) as ex:
            list(ex.map(run, [[HIPCC, *compile_flags, *SOURCE_FLAGS.get(os.path.basename(src), []), "-c", src,
                               "-o", obj] for src, obj in zip(SOURCES, objs)]))
        tmp = out + ".tmp%d" % os.getpid()
        run([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", *objs, "-o", tmp])
        os.replace(tmp, out)
    finally:
        for o in objs:
            if os.path.exists(o):
                os.remove(o)
        if os.path.isdir(objdir):
            os.rmdir(objdir)
    return out


if __name__ == "__main__":
    print(build(verbose=True))
    print(build_probe(verbose=True))
    print(build_binding(verbose=True))
