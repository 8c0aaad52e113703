"""Build libbevpool.so for gfx950 with hipcc, in-tree, and, where there is a ROCm build of
torch, the native module _layer_native.so that calls it on torch tensors.

``python -m paper_2205_13542_amd.build`` (or ``build()``) always recompiles,
so a stale library never survives a source change.
"""
from __future__ import annotations

import os
import shutil
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIB_PATH = os.path.join(HERE, "libbevpool.so")
# measurement probe for bench.py --floor (not part of the pooling library)
FLOOR_SOURCE = "floor.hip"
FLOOR_LIB_PATH = os.path.join(HERE, "libbevpool_floor.so")
# calls of libbevpool.so on torch tensors, for layer_ops.py; host code alone
TORCH_SOURCE = "layer_torch.cpp"
TORCH_LIB_PATH = os.path.join(HERE, "_layer_native.so")
SOURCES = ["bevpool.hip", "plan.hip", "forward.hip", "backward.hip", "layout.hip",
           "mapops.hip", "norm.hip", "dropout.hip", "attention.hip",
           "attention_backward.hip", "layerops.hip", "rms_norm.hip", "rotary.hip",
           "gated.hip", "linear_int8.hip"]

CXX = os.environ.get("CXX", "g++")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = [
    "-O3", "-std=c++17", "--offload-arch=gfx950", "-fPIC", "-shared",
    # bit-exact plan geometry: no contraction into fused multiply-adds
    "-ffp-contract=off",
    # no packed fp32 instructions in generated code
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function",
    "-fvisibility=hidden",
]


def _torch_commands(lib_dir: str, tmp: str) -> list:
    """Compile and link commands of the native module; none where there is no ROCm build of torch, or no
    compiler or Python headers, which only the module needs."""
    import importlib.util
    import sysconfig
    import warnings
    spec = importlib.util.find_spec("torch")
    if spec is None or spec.origin is None:
        return []
    torch_dir = os.path.dirname(spec.origin)
    if not os.path.exists(os.path.join(torch_dir, "lib", "libtorch_hip.so")):
        return []
    python = sysconfig.get_paths()["include"]
    missing = CXX if shutil.which(CXX) is None else "Python.h"
    if missing == CXX or not os.path.exists(os.path.join(python, "Python.h")):
        warnings.warn(f"no {missing}: {os.path.basename(TORCH_LIB_PATH)} is left out, which layer_ops needs")
        return []
    obj = tmp + ".o"
    rocm = os.path.dirname(os.path.dirname(os.path.realpath(HIPCC)))
    system = [os.path.join(torch_dir, "include"), os.path.join(torch_dir, "include", "torch", "csrc", "api", "include"),
              os.path.join(rocm, "include"), python]
    compile_ = [CXX, "-O2", "-std=c++17", "-fPIC", "-fvisibility=hidden", "-Wall", "-D__HIP_PLATFORM_AMD__=1",
                "-DUSE_ROCM=1", "-I", INCLUDE, *(a for d in system for a in ("-isystem", d)), "-c",
                os.path.join(CSRC, TORCH_SOURCE), "-o", obj]
    link = [CXX, "-shared", obj, "-o", tmp, "-L", lib_dir, "-lbevpool", "-L", os.path.join(torch_dir, "lib"),
            *("-l" + name for name in ("c10", "c10_hip", "torch_cpu", "torch_hip", "torch", "torch_python")),
            "-Wl,-rpath,$ORIGIN"]
    return [compile_, link]


def _run(command) -> None:
    done = subprocess.run(command, capture_output=True, text=True)
    if done.returncode != 0:
        raise subprocess.CalledProcessError(done.returncode, done.args, done.stdout, done.stderr)


def _install(made: str, path: str) -> None:
    shutil.copy(made, path + ".tmp")        # the folders may be on two file systems
    os.replace(path + ".tmp", path)


def build(verbose: bool = False) -> str:
    """Compile every source to an object in parallel, then link and install the library, then the module.

    Where the module is not built, or fails to, the library is installed all the same and no
    older module is left beside it; a failure is raised then."""
    import concurrent.futures
    import tempfile
    compile_flags = [f for f in FLAGS if f != "-shared"]
    with tempfile.TemporaryDirectory(prefix="bevpool_build_") as tmpdir:
        objs = [os.path.join(tmpdir, os.path.splitext(s)[0] + ".o") for s in SOURCES]
        cmds = [[HIPCC, *compile_flags, "-I", INCLUDE, "-I", CSRC, "-c",
                 os.path.join(CSRC, s), "-o", o] for s, o in zip(SOURCES, objs)]
        floor_tmp, lib_tmp, torch_tmp = (os.path.join(tmpdir, os.path.basename(p))
                                         for p in (FLOOR_LIB_PATH, LIB_PATH, TORCH_LIB_PATH))
        cmds.append([HIPCC, *FLAGS, os.path.join(CSRC, FLOOR_SOURCE), "-o", floor_tmp])
        torch_cmds = _torch_commands(tmpdir, torch_tmp)
        if verbose:
            for c in cmds + torch_cmds[:1]:
                print(" ".join(c), flush=True)
        workers = max(1, min(len(cmds) + 1, os.cpu_count() or 1))
        with concurrent.futures.ThreadPoolExecutor(workers) as ex:
            module = ex.submit(_run, torch_cmds[0]) if torch_cmds else None
            for r in [ex.submit(_run, c) for c in cmds]:
                r.result()
        _run([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", *objs, "-o", lib_tmp])
        _install(floor_tmp, FLOOR_LIB_PATH)
        _install(lib_tmp, LIB_PATH)
        try:
            if module:
                module.result()
                _run(torch_cmds[1])
                _install(torch_tmp, TORCH_LIB_PATH)
        finally:
            if not os.path.exists(torch_tmp) and os.path.exists(TORCH_LIB_PATH):
                os.remove(TORCH_LIB_PATH)       # one of another library
    return LIB_PATH


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
