"""Build libgpuos.so (HIP kernels + host runtime) for gfx950 and, where PyTorch is installed, _binding.so (the module on its tensors), in-tree."""
import importlib.util
import os
import subprocess
import sys
import sysconfig
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libgpuos.so")
BINDING, BINDING_SOURCE = os.path.join(HERE, "_binding.so"), os.path.join(CSRC, "gpuos_binding.cpp")
SOURCES = ["gpuos_kernels.hip", "gpuos_model.hip", "gpuos_cache.hip", "gpuos_runtime.cpp", "gpuos_model.cpp", "gpuos_cache.cpp", "gpuos_jit.cpp"]
HEADERS = ["gpuos_internal.h", "gpuos_device.h", "gpuos_model.h", "gpuos_model_device.h", "gpuos_cache.h", "gpuos_on_device.h", os.path.join("..", "..", "include", "gpuos.h")]

# -ffp-contract=off: only the FMA operator fuses.  The -packed-fp32-ops target feature switch
# keeps the compiler from forming packed fp32 instructions.
FLAGS = ["-O3", "--offload-arch=gfx950", "-std=c++17", "-fPIC", "-shared", "-ffp-contract=off",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-Wall", "-Wno-unused-variable",
         "-Wno-unused-but-set-variable", "-pthread", "-DGPUOS_CSRC_DIR=" + CSRC, "-ldl"]


def _older(made, deps):
    return not os.path.exists(made) or any(os.path.getmtime(d) > os.path.getmtime(made) for d in deps)


def needs_build():
    return (_older(LIB, [os.path.join(CSRC, s) for s in SOURCES + HEADERS] + [os.path.abspath(__file__)])
            or has_torch() and _older(BINDING, [BINDING_SOURCE, os.path.join(CSRC, HEADERS[-1]), os.path.abspath(__file__)]))


def has_torch():
    return importlib.util.find_spec("torch") is not None


def binding_command():
    """The host compiler's command for the module, against the headers and libraries of the PyTorch that is installed."""
    import torch
    home = os.path.dirname(torch.__file__)
    include = [os.path.join(home, "include"), os.path.join(home, "include", "torch", "csrc", "api", "include"), sysconfig.get_paths()["include"]]
    return (["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall", "-D_GLIBCXX_USE_CXX11_ABI=%d" % torch.compiled_with_cxx11_abi()] + ["-isystem" + i for i in include]
            + ["-o", BINDING, BINDING_SOURCE, "-L" + os.path.join(home, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10"])


def _all(jobs):
    """Run commands beside each other: what they say, or the first that failed as an exception."""
    running = [subprocess.Popen(j, cwd=CSRC, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True) for j in jobs]
    said = [r.communicate()[0] for r in running]
    out = ["\n".join(l for l in t.splitlines() if "packed-fp32-ops" not in l) for t in said]
    for r, t in zip(running, out):
        if r.returncode != 0:
            raise RuntimeError(os.path.basename(r.args[0]) + " failed:\n" + t)
    return "\n".join(t for t in out if t.strip())


def build(force=True, verbose=False):
    if not force and not needs_build():
        return LIB
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    flags = (["-Rpass-analysis=kernel-resource-usage"] if verbose else []) + [f for f in FLAGS if f not in ("-shared", "-ldl")]
    with tempfile.TemporaryDirectory() as made, ThreadPoolExecutor(1) as beside:      # (a source at a time would take as long as all of them: two to four minutes)
        module = beside.submit(lambda: _all([binding_command()])) if has_torch() else None
        objects = [os.path.join(made, s + ".o") for s in SOURCES]
        jobs = [[hipcc] + flags + ["-c", "-o", o, os.path.join(CSRC, s)] for s, o in zip(SOURCES, objects)]
        out = _all(jobs) + _all([[hipcc, "--offload-arch=gfx950", "-shared", "-pthread", "-o", LIB] + objects + ["-ldl"]])
        if module:                                              # (whatever becomes of it, the library is there)
            out += module.result()
    if verbose or out.strip():
        print(out, file=sys.stderr)
    return LIB


if __name__ == "__main__":
    build(force=True, verbose="-v" in sys.argv)
    print(LIB)
