"""Builds libpahq.so (HIP, gfx950 only) in-tree with hipcc, and _tensors.so, the torch side of its operators on device tensors."""
import importlib.util
import os
import re
import shutil
import subprocess
import sysconfig
import warnings
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libpahq.so")
EXTENSION = os.path.join(HERE, "_tensors.so")
SOURCES = ["rows.hip", "gemm.hip", "oproj.hip", "attn_kl.hip", "engine.hip", "api.hip", "ceilings.hip", "noalloc.hip", "mx4.hip",
           "rotary.hip", "kv_cache.hip", "kv_attention.hip"]
# -ffp-contract=off: a product and a sum are rounded separately unless the source says fmaf.  The same
# expression (a norm's x * rstd * gain + offset, a GEMM epilogue's acc * scale + bias) is compiled into
# several kernels -- cache passes and candidate passes take different ones -- and results that must agree
# bit for bit between them (a clean patch scores exactly 0) may not depend on where the compiler chose to fuse.
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-ffp-contract=off",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]


# Kernels that may not keep registers in scratch memory: their waits count the memory operations that they have in flight themselves, and
# one that spilled on its way to its addresses would reach memory with what it read back.
NO_SCRATCH = {"kv_cache.hip", "kv_attention.hip"}
RESOURCES = "-Rpass-analysis=kernel-resource-usage"


def scratch_of(remarks):
    """{kernel: bytes of scratch a lane} of the kernels that have any, from what the compiler says with RESOURCES."""
    found = re.findall(r"Function Name: (\S+)|ScratchSize \[bytes/lane\]: (\d+)|(Dynamic Stack: True)", remarks)
    out, name = {}, None
    for function, size, stack in found:
        name = function or name
        if stack or int(size or 0):
            out[name] = int(size or 0)
    return out


def _compile(src):
    obj = os.path.join(HERE, "_build", src.replace(".hip", ".o"))
    said = subprocess.run(["hipcc", *FLAGS, *([RESOURCES] if src in NO_SCRATCH else []), "-c", os.path.join(CSRC, src), "-o", obj], check=True,
                          stdout=subprocess.PIPE, stderr=subprocess.STDOUT)
    if src in NO_SCRATCH and said is not None:
        remarks = said.stdout.decode(errors="replace")
        spilled = scratch_of(remarks)
        if spilled or "ScratchSize" not in remarks:
            os.remove(obj)
            raise RuntimeError("%s: kernels with registers in scratch memory: %s" % (src, spilled or "the compiler does not say"))
    return obj


def _extension():
    """csrc/tensors_ext.cpp against torch's and Python's headers; torch's libraries are there when tensors.py loads it.  libpahq.so
    needs none of them: where one is missing it is left without the extension, and tensors.py says so when it is used."""
    spec = importlib.util.find_spec("torch")
    torch = os.path.dirname(spec.origin) if spec else ""
    missing = [what for what, there in (("torch", spec), ("torch's headers", spec and os.path.isdir(os.path.join(torch, "include", "ATen"))),
                                        ("Python's headers", os.path.exists(os.path.join(sysconfig.get_paths()["include"], "Python.h"))),
                                        ("g++", shutil.which("g++"))) if not there]
    if missing:
        if os.path.exists(EXTENSION):                       # one that was built for another libpahq.so
            os.remove(EXTENSION)
        warnings.warn("no operators on device tensors (_tensors.so): without " + ", ".join(missing))
        return
    subprocess.run(["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-D__HIP_PLATFORM_AMD__=1", "-DUSE_ROCM=1", "-I" + os.path.join(torch, "include"),
                    "-I" + os.path.join(torch, "include", "torch", "csrc", "api", "include"), "-I/opt/rocm/include", "-I" + sysconfig.get_paths()["include"],
                    os.path.join(CSRC, "tensors_ext.cpp"), "-o", EXTENSION, "-L" + HERE, "-l:libpahq.so", "-L" + os.path.join(torch, "lib"),
                    "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_hip", "-L/opt/rocm/lib", "-lamdhip64", "-Wl,-rpath,$ORIGIN"],
                   check=True, stdout=subprocess.PIPE, stderr=subprocess.STDOUT)


def build(verbose=False):
    os.makedirs(os.path.join(HERE, "_build"), exist_ok=True)
    with ThreadPoolExecutor(max_workers=6) as ex:
        objs = list(ex.map(_compile, SOURCES))
    subprocess.run(["hipcc", "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB, *objs], check=True,
                   stdout=subprocess.PIPE, stderr=subprocess.STDOUT)
    _extension()
    if verbose:
        print("built", LIB)
    return LIB


if __name__ == "__main__":
    build(verbose=True)
