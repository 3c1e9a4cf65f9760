"""Build libgpuos.so (HIP kernels + host runtime) for gfx950, in-tree."""
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libgpuos.so")
SOURCES = ["gpuos_kernels.hip", "gpuos_model.hip", "gpuos_cache.hip", "gpuos_runtime.cpp", "gpuos_model.cpp", "gpuos_cache.cpp", "gpuos_jit.cpp"]
HEADERS = ["gpuos_internal.h", "gpuos_device.h", "gpuos_model.h", "gpuos_model_device.h", "gpuos_cache.h", "gpuos_on_device.h", os.path.join("..", "..", "include", "gpuos.h")]

# -ffp-contract=off: only the FMA operator fuses.  The -packed-fp32-ops target feature switch
# keeps the compiler from forming packed fp32 instructions.
FLAGS = ["-O3", "--offload-arch=gfx950", "-std=c++17", "-fPIC", "-shared", "-ffp-contract=off",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-Wall", "-Wno-unused-variable",
         "-Wno-unused-but-set-variable", "-pthread", "-DGPUOS_CSRC_DIR=" + CSRC, "-ldl"]


def needs_build():
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = [os.path.join(CSRC, s) for s in SOURCES + HEADERS] + [os.path.abspath(__file__)]
    return any(os.path.getmtime(d) > t for d in deps)


def build(force=True, verbose=False):
    if not force and not needs_build():
        return LIB
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    cmd = [hipcc] + FLAGS + ["-o", LIB] + [os.path.join(CSRC, s) for s in SOURCES]
    if verbose:
        cmd.insert(1, "-Rpass-analysis=kernel-resource-usage")
    r = subprocess.run(cmd, cwd=CSRC, capture_output=True, text=True)
    out = "\n".join(l for l in (r.stdout + r.stderr).splitlines() if "packed-fp32-ops" not in l)
    if r.returncode != 0:
        raise RuntimeError("hipcc failed:\n" + out)
    if verbose or out.strip():
        print(out, file=sys.stderr)
    return LIB


if __name__ == "__main__":
    build(force=True, verbose="-v" in sys.argv)
    print(LIB)
