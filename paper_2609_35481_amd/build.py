"""Build the planner's HIP library for gfx950 (in-tree shared object)."""
from __future__ import annotations

import os
import shutil
import subprocess
import sysconfig
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
SRCS = [os.path.join(HERE, "csrc", n) for n in ("topoep.hip", "layout.hip", "gather.hip", "router.hip", "moe.hip", "grads.hip",
                                              "rows.hip", "ffn.hip", "int8.hip")]
SRC = SRCS[0]
LIB = os.path.join(HERE, "libtopoep.so")
INCLUDE = os.path.join(ROOT, "include")

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    # no packed-FP32 instructions in any generated code
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
]


# The same library with phase stamps (-DTOPOEP_STAMPS): the solver and the
# first chunk write the wall clock at phase boundaries into the workspace's
# control words.  For measurement only (bench.py --phases); the product
# library is LIB.
STAMPS_LIB = os.path.join(HERE, "libtopoep_stamps.so")

# The binding's calls over torch's C++ tensors, Python modules.
TENSORS_SRC = os.path.join(HERE, "csrc", "tensors.cpp")
TENSORS_LIB = os.path.join(HERE, "_tensors.so")
FFN_TENSORS_SRC = os.path.join(HERE, "csrc", "ffn_tensors.cpp")
FFN_TENSORS_LIB = os.path.join(HERE, "_ffn_tensors.so")


def _tensors_command(out: str, src: str, extra=()) -> list:
    import torch
    base = os.path.dirname(torch.__file__)
    include = os.path.join(base, "include")
    return [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-w",
            "-D_GLIBCXX_USE_CXX11_ABI=%d" % int(torch._C._GLIBCXX_USE_CXX11_ABI), "-I", INCLUDE, "-I", include, "-I",
            os.path.join(include, "torch", "csrc", "api", "include"), "-I", sysconfig.get_paths()["include"],
            *extra, "-o", out, src, "-L", os.path.join(base, "lib"), "-ltorch_python", "-ltorch_cpu", "-ltorch",
            "-lc10", *(["-lc10_hip", "-ltorch_hip"] if extra else [])]


def _run_all(commands, verbose: bool) -> None:
    """Run the commands side by side; raise with the output of those that failed."""
    procs = [(cmd, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.PIPE, text=True)) for cmd in commands]
    errors = []
    for cmd, proc in procs:
        so, se = proc.communicate()
        if proc.returncode != 0:
            errors.append("%s failed:\n%s%s" % (" ".join(cmd), so, se))
        elif verbose:
            print(se)
    if errors:
        raise RuntimeError("\n".join(errors))


def build(verbose: bool = False) -> str:
    """Compile every source (processes side by side), then link LIB and
    STAMPS_LIB, which differ in the planner's object alone, and the binding's
    two modules."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    with tempfile.TemporaryDirectory() as tmp:
        def compiled(src, name, *extra):
            return [hipcc, *HIPCC_FLAGS, *extra, "-I", INCLUDE, "-c", "-o", os.path.join(tmp, name), src]

        objects = {src: os.path.basename(src) + ".o" for src in SRCS}
        tensors, ffn_tensors = os.path.join(tmp, "_tensors.so"), os.path.join(tmp, "_ffn_tensors.so")
        hip = ["-D__HIP_PLATFORM_AMD__=1", "-DUSE_ROCM", "-I", "/opt/rocm/include"]   # torch's streams
        _run_all([compiled(src, name) for src, name in objects.items()] +
                 [compiled(SRC, "stamps.o", "-DTOPOEP_STAMPS"), _tensors_command(tensors, TENSORS_SRC),
                  _tensors_command(ffn_tensors, FFN_TENSORS_SRC, hip)], verbose)
        links = []
        for out, planner in ((LIB, objects[SRC]), (STAMPS_LIB, "stamps.o")):
            parts = [planner if src == SRC else name for src, name in objects.items()]
            links.append((out, os.path.join(tmp, os.path.basename(out)), [os.path.join(tmp, p) for p in parts]))
        _run_all([[hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", made, *parts] for _, made, parts in links],
                 verbose)
        for out, made in [(out, made) for out, made, _ in links] + [(TENSORS_LIB, tensors), (FFN_TENSORS_LIB, ffn_tensors)]:
            fresh = out + ".tmp%d" % os.getpid()
            shutil.copy(made, fresh)
            os.replace(fresh, out)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
