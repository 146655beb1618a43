"""Build step for the HIP library ``libedkm.so`` (gfx950), in-tree."""
from __future__ import annotations

import os
import subprocess
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
# The clustering's sources, which the diagnostics and test builds compile with flags of
# their own, and the layer and optimizer operators', which all builds share.
SOURCES = [os.path.join(CSRC, f) for f in ("edkm_kernels.hip", "edkm_api.hip")]
LAYER_SOURCES = [os.path.join(CSRC, f) for f in ("edkm_product.hip", "edkm_product_palette.hip", "edkm_few.hip", "edkm_adamw.hip",
                                                      "edkm_layer_api.hip", "edkm_embedding.hip", "edkm_norm.hip", "edkm_loss.hip",
                                                      "edkm_loss_products.hip", "edkm_model_api.hip")]
OUT = os.path.join(HERE, "libedkm.so")
# Diagnostics build: the same library with per-block timeline stamps
# (-DEDKM_BLOCK_STAMPS, include/edkm_stamps.h); load it with EDKM_LIBRARY.
OUT_STAMPS = os.path.join(HERE, "libedkm_stamps.so")
# Test build: no block of a table phase waits for another one's rows, and every
# second block starts late (tests/test_gpu_exchange.py).
OUT_EXCHANGE = os.path.join(HERE, "libedkm_exchange.so")

# Marshalling of the layer and optimizer calls for torch tensors (a Python extension).
OUT_BINDING = os.path.join(HERE, "_edkm_torch.so")

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Werror=uninitialized",
    # no packed-fp32 instructions in generated code
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-I" + os.path.join(ROOT, "include"),
]


def _hipcc(args):
    subprocess.check_call([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), *args])


def _compile(folder, jobs):
    """Objects of (source, extra flags) pairs, side by side."""
    def one(job):
        i, (src, extra) = job
        obj = os.path.join(folder, "%d_%s.o" % (i, os.path.basename(src)))
        _hipcc([*HIPCC_FLAGS, *extra, "-c", src, "-o", obj])
        return obj
    with ThreadPoolExecutor(min(8, os.cpu_count() or 1)) as pool:
        return list(pool.map(one, enumerate(jobs)))


def _link(out, objects):
    tmp = out + ".tmp%d" % os.getpid()
    _hipcc(["--offload-arch=gfx950", "-shared", "-fPIC", "-o", tmp, *objects])
    os.replace(tmp, out)
    return out


STAMPS_FLAGS = ("-DEDKM_BLOCK_STAMPS",)
EXCHANGE_FLAGS = ("-DEDKM_XW_WAIT=-1", "-DEDKM_XW_LATE=300000")


def build_libraries(builds) -> list:
    """Each (output, extra flags) build of the library; what they share is compiled once."""
    with tempfile.TemporaryDirectory() as folder:
        jobs = [(s, ()) for s in LAYER_SOURCES] + [(s, tuple(extra)) for _, extra in builds for s in SOURCES]
        objs = _compile(folder, jobs)
        shared, own = objs[:len(LAYER_SOURCES)], objs[len(LAYER_SOURCES):]
        n = len(SOURCES)
        return [_link(out, own[n * i:n * i + n] + shared) for i, (out, _) in enumerate(builds)]


def build_library(out: str = OUT, extra=()) -> str:
    return build_libraries([(out, extra)])[0]


def build_stamps(out: str = OUT_STAMPS) -> str:
    return build_library(out, extra=STAMPS_FLAGS)


def build_exchange(out: str = OUT_EXCHANGE) -> str:
    return build_library(out, extra=EXCHANGE_FLAGS)


def build_all() -> list:
    """The product library, its diagnostics and test builds, and the marshalling."""
    return [build_binding()] + build_libraries([(OUT, ()), (OUT_STAMPS, STAMPS_FLAGS), (OUT_EXCHANGE, EXCHANGE_FLAGS)])


def build_binding(out: str = OUT_BINDING) -> str:
    """The compiled marshalling for torch tensors (host code only)."""
    import sysconfig
    import torch
    root = os.path.dirname(torch.__file__)
    inc = [os.path.join(root, "include"), os.path.join(root, "include", "torch", "csrc", "api", "include"),
           sysconfig.get_paths()["include"], "/opt/rocm/include"]
    tmp = out + ".tmp%d" % os.getpid()
    subprocess.check_call(["g++", "-std=c++17", "-O2", "-fPIC", "-shared", "-fvisibility=hidden", "-Wall",
                           "-D__HIP_PLATFORM_AMD__=1", "-DUSE_ROCM=1",
                           "-D_GLIBCXX_USE_CXX11_ABI=%d" % torch._C._GLIBCXX_USE_CXX11_ABI,
                           *[a for i in inc for a in ("-isystem", i)], "-o", tmp, os.path.join(HERE, "csrc", "edkm_torch.cpp"),
                           "-L" + os.path.join(root, "lib"), "-ltorch_python", "-ltorch", "-ltorch_cpu", "-lc10", "-lc10_hip"])
    os.replace(tmp, out)
    return out


if __name__ == "__main__":
    print("\n".join(build_all()))
