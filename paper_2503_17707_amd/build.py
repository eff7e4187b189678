"""Build libpipeboost.so for gfx950 with hipcc (in-tree, no JIT cache).

Every HIP source is compiled with packed FP32 instructions disabled
(``-Xclang -target-feature -Xclang -packed-fp32-ops``); hipcc's host pass
warns that it does not know the feature, which is harmless.
"""
import concurrent.futures as cf
import hashlib
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
# the paged cache and beam search, apart from the model's kernels: profile summaries
# hold for the contents of csrc
PAGED = os.path.join(HERE, "paged")
Q8 = os.path.join(HERE, "q8")  # 8-bit linear layers
OUT_DIR = os.path.join(HERE, "lib")
LIB = os.path.join(OUT_DIR, "libpipeboost.so")
SOURCES = ["gemm.hip", "attention.hip", "misc.hip", "lmhead.hip", "model.cpp", "sched.cpp"]
PAGED_SOURCES = ["paged_attention.hip", "paged_cache.hip", "beam.hip", "paged_ops.cpp"]
Q8_SOURCES = ["gemm_q8.hip", "rows_q8.hip", "q8_ops.cpp"]
ARGS = os.path.join(OUT_DIR, "pipeboost_q8_args.so")
ARCH = os.environ.get("PB_OFFLOAD_ARCH", "gfx950")
FLAGS = ["-O3", "-std=c++17", "-fPIC", "--offload-arch=" + ARCH, "-Wall", "-Wno-unused-result",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-I" + os.path.join(ROOT, "include"), "-I" + CSRC]


def _compile(src: str, obj_dir: str, defines=()) -> str:
    obj = os.path.join(obj_dir, os.path.splitext(src)[0] + ".o")
    lang = ["-x", "hip"] if src.endswith(".cpp") else []
    path = os.path.join(PAGED if src in PAGED_SOURCES else Q8 if src in Q8_SOURCES else CSRC, src)
    cmd = (["hipcc", "-c"] + lang + [path, "-o", obj] + FLAGS
           + ["-D" + d for d in defines])
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("compile of %s failed:\n%s\n%s" % (src, " ".join(cmd), r.stderr))
    noise = [ln for ln in r.stderr.splitlines() if "packed-fp32-ops" not in ln and ln.strip()]
    if noise:
        sys.stderr.write("\n".join(noise) + "\n")
    return obj


def build_args() -> str:
    """The extension module that looks over the 8-bit operators' tensors (host code, torch's headers)."""
    import sysconfig

    import torch
    from torch.utils.cpp_extension import ROCM_HOME, include_paths, library_paths

    os.makedirs(OUT_DIR, exist_ok=True)
    tmp = ARGS + ".tmp%d" % os.getpid()
    cmd = (["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden", "-Wall", "-D__HIP_PLATFORM_AMD__=1",
            "-DUSE_ROCM=1", "-D_GLIBCXX_USE_CXX11_ABI=%d" % torch._C._GLIBCXX_USE_CXX11_ABI,
            '-DPB_TORCH="%s"' % torch.__version__, os.path.join(Q8, "py_q8.cpp"), "-o", tmp]
           + ["-isystem" + d for d in include_paths() + [sysconfig.get_paths()["include"], os.path.join(ROCM_HOME or "/opt/rocm", "include")]]
           + ["-L" + d for d in library_paths()] + ["-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_hip"])
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("compile of py_q8.cpp failed:\n%s\n%s" % (" ".join(cmd), r.stderr))
    os.replace(tmp, ARGS)
    return ARGS


def _try_args():
    """build_args where it can be built: the library does without it, and programs of the C ABI without torch."""
    try:
        build_args()
    except Exception as e:
        if os.path.exists(ARGS):
            os.remove(ARGS)  # an older one would be called with newer arguments
        sys.stderr.write("%s was not built (the 8-bit operators' Python wrappers need it): %s\n" % (os.path.basename(ARGS), e))


def build(verbose: bool = False, out: str = LIB, defines=()) -> str:
    """Compile and link; `out` and `defines` (NAME=VALUE) select a variant build."""
    tag = hashlib.md5(repr((out, tuple(defines))).encode()).hexdigest()[:10]
    obj_dir = os.path.join(ROOT, "_build", "pipeboost_" + tag)
    os.makedirs(obj_dir, exist_ok=True)
    os.makedirs(os.path.dirname(out), exist_ok=True)
    sources = SOURCES + PAGED_SOURCES + Q8_SOURCES
    with cf.ThreadPoolExecutor(max_workers=min(8, len(sources))) as ex:
        if out == LIB:
            ex.submit(_try_args)
        objs = list(ex.map(lambda s: _compile(s, obj_dir, defines), sources))
    tmp = out + ".tmp%d" % os.getpid()
    cmd = ["hipcc", "-shared", "-fPIC", "--offload-arch=" + ARCH, "-o", tmp] + objs
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("link failed:\n%s\n%s" % (" ".join(cmd), r.stderr))
    os.replace(tmp, out)
    if verbose:
        print("built", out)
    return out


if __name__ == "__main__":
    build(verbose=True)
