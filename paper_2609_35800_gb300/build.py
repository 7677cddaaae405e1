"""Build the HeadGuard C-ABI library (libheadguard.so) for sm_103a, in-tree.

Each .cu translation unit is compiled by its own nvcc process (in parallel)
and the objects are linked into paper_2609_35800_gb300/_build/libheadguard.so
with the CUDA runtime linked statically.  No FMA contraction is forbidden
globally: the kernels that decide stored bits use explicit round-to-nearest
intrinsics instead.
"""
import concurrent.futures
import os
import shutil
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
CSRC_ATTENTION = os.path.join(HERE, "csrc_attention")  # caches that stay 16-bit, prompt attention
INCLUDE = os.path.join(ROOT, "include")
OUT_DIR = os.path.join(HERE, "_build")
LIB_NAME = "libheadguard.so"
LIB = os.path.join(OUT_DIR, LIB_NAME)
SOURCES = [os.path.join(CSRC, f) for f in ("hg_api.cu", "hg_quantize.cu", "hg_decode.cu", "hg_decode_m16.cu",
                                            "hg_noalloc.cu")]
SOURCES += [os.path.join(CSRC_ATTENTION, f) for f in ("hg_pages_api.cu", "hg_pages_append.cu", "hg_pages_decode.cu",
                                                      "hg_prompt.cu")]
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
NVCC_FLAGS = ["-O3", "-lineinfo", "-std=c++17", "-Xcompiler", "-fPIC", "-Xcompiler", "-Wall",
              "-I" + INCLUDE, "-I" + CSRC, "-I" + CSRC_ATTENTION]


def nvcc():
    path = shutil.which("nvcc")
    if path:
        return path
    cand = "/usr/local/cuda/bin/nvcc"
    if os.path.exists(cand):
        return cand
    raise RuntimeError("nvcc not found")


def _inputs():
    files = [os.path.join(d, f) for d in (CSRC, CSRC_ATTENTION) for f in os.listdir(d)]
    files.append(os.path.join(INCLUDE, "headguard.h"))
    files.append(os.path.abspath(__file__))
    return files


def _stale():
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    return any(os.path.getmtime(f) > t for f in _inputs())


def _compile(src, extra):
    obj = os.path.join(OUT_DIR, os.path.splitext(os.path.basename(src))[0] + ".o")
    cmd = [nvcc()] + ARCH + NVCC_FLAGS + extra + ["-c", src, "-o", obj]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("nvcc failed for %s:\n%s\n%s" % (src, " ".join(cmd), res.stderr))
    return obj, res.stderr


def build(force=False, verbose=False, extra_flags=()):
    """Compile and link libheadguard.so; return its path."""
    if not force and not _stale():
        return LIB
    os.makedirs(OUT_DIR, exist_ok=True)
    with concurrent.futures.ThreadPoolExecutor(max_workers=len(SOURCES)) as ex:
        results = list(ex.map(lambda s: _compile(s, list(extra_flags)), SOURCES))
    if verbose:
        for _, err in results:
            if err:
                print(err)
    tmp = LIB + ".tmp.%d" % os.getpid()
    cmd = [nvcc()] + ARCH + ["-shared", "-o", tmp] + [o for o, _ in results]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("link failed:\n%s" % res.stderr)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    import sys
    print(build(force=True, verbose="-v" in sys.argv,
                extra_flags=["-Xptxas", "-v"] if "-v" in sys.argv else []))
