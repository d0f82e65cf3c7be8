"""Builds the HIP library libpictura.so for gfx950 and the binding's helper
_tensors.so (in-tree)."""
import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(os.path.dirname(HERE), "include")
LIB = os.path.join(HERE, "libpictura.so")
TENSORS = os.path.join(HERE, "_tensors.so")
SOURCES = ["pictura_binner.hip", "pictura_render.hip", "pictura_encoder.hip", "pictura_policy.hip", "pictura_adamw.hip",
           "pictura_memory.hip", "pictura_norm.hip", "pictura_prefer.hip",
           "pictura_abi.hip"]
# (source, object name, extra flags): the render source is compiled three
# times.  One object holds only the production class/depth kernels, one the
# production instance and one-sample colour kernels, both scheduled by LLVM's
# iterative ILP strategy (1.4 % faster on the class/depth kernel, and 1.6 %
# and 2.5 % on the tile-shape-specialised instance and colour kernels, than
# the next best setting, in A/B runs with identical images); the antialiased
# kernel spills and slows under it, so it keeps the default scheduler.
# The policy source is compiled once for the entries and once for the kernels of
# each type of logits, side by side.
UNITS = [(src, src.replace(".hip", ".o"), []) for src in SOURCES] + [
    ("pictura_policy.hip", f"pictura_policy_{name}.o", [f"-DPICTURA_POLICY_TYPE={kind}"])
    for name, kind in (("f32", "float"), ("bf16", "__bf16"), ("f16", "_Float16"))] + [
    ("pictura_render.hip", "pictura_render_plain.o",
     ["-DPICTURA_RENDER_PLAIN", "-mllvm", "-amdgpu-sched-strategy=iterative-ilp"]),
    ("pictura_render.hip", "pictura_render_side.o",
     ["-DPICTURA_RENDER_SIDE", "-mllvm", "-amdgpu-sched-strategy=iterative-ilp"]),
]

# fp32 rules need IEEE arithmetic: no contraction, correctly rounded division,
# denormals kept.  Packed fp32 instructions are disabled.
HIPCC_FLAGS = [
    "-O3", "-std=c++17", "--offload-arch=gfx950", "-fPIC",
    "-ffp-contract=off", "-fno-fast-math", "-fhip-fp32-correctly-rounded-divide-sqrt",
    "-fno-gpu-flush-denormals-to-zero",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function",
]


def _tensors_command(out: str) -> list:
    """The host compiler's command for the helper that reads torch tensors and makes the calls that take them."""
    import sysconfig

    import torch
    root = os.path.dirname(torch.__file__)
    inc = os.path.join(root, "include")
    rocm = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "include")
    return [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall", "-Wno-unused-function",
            "-D__HIP_PLATFORM_AMD__", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch.compiled_with_cxx11_abi())}", "-isystem", inc,
            "-isystem", os.path.join(inc, "torch", "csrc", "api", "include"), "-isystem", rocm, "-I", INCLUDE, "-I",
            sysconfig.get_paths()["include"], os.path.join(CSRC, "pictura_tensors.cpp"),
            os.path.join(CSRC, "pictura_calls.cpp"), "-o", out, "-L", os.path.join(root, "lib"), "-ltorch_python", "-ltorch",
            "-ltorch_cpu", "-lc10", "-lc10_hip"]


def build(verbose: bool = False) -> str:
    """Builds both.  The helper alone needs a host compiler and torch's C++ headers: without
    them this raises once the library is there, with which the renderer and the encoder run."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    objs, procs = [], []
    try:
        tensors = _tensors_command(TENSORS + ".tmp")
        if verbose:
            print(" ".join(tensors))
        helper = subprocess.Popen(tensors)
    except (ImportError, OSError) as e:
        helper, missing = None, e
    for src, oname, extra in UNITS:
        obj = os.path.join(CSRC, oname)
        cmd = [hipcc, *HIPCC_FLAGS, *extra, "-I", INCLUDE, "-c", os.path.join(CSRC, src), "-o", obj]
        if verbose:
            print(" ".join(cmd))
        procs.append(subprocess.Popen(cmd))
        objs.append(obj)
    for p in procs:
        if p.wait() != 0:
            raise RuntimeError(f"{p.args[0]} failed")
    tmp = LIB + ".tmp"
    subprocess.check_call([hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", "-Wl,--no-undefined", "-o", tmp, *objs])
    os.replace(tmp, LIB)
    for o in objs:
        os.remove(o)
    if helper is None or helper.wait() != 0:
        raise RuntimeError(f"{LIB} is built; {TENSORS}, which the policy's operators need, is not: " +
                           (str(missing) if helper is None else f"{tensors[0]} failed"))
    os.replace(TENSORS + ".tmp", TENSORS)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
