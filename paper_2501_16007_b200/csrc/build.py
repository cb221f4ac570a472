"""Builds csrc/libtoploc.so for sm_100a with nvcc (cross-compiles without a GPU).

    python -m paper_2501_16007_b200.csrc.build [--force] [--verbose]
"""
import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

_HERE = os.path.dirname(os.path.abspath(__file__))
_ROOT = os.path.dirname(os.path.dirname(_HERE))
_INCLUDE = os.path.join(_ROOT, "include")
PROOF_SOURCES = [os.path.join(_HERE, "toploc.cu"), os.path.join(_HERE, "toploc_direct.cu"),
                 os.path.join(_HERE, "toploc_producer.cu")]
MODEL_SOURCES = [os.path.join(_HERE, "toploc_pages.cu"), os.path.join(_HERE, "toploc_norm.cu"),
                 os.path.join(_HERE, "toploc_attention.cu"), os.path.join(_HERE, "toploc_attention_tc.cu"),
                 os.path.join(_HERE, "toploc_attention_few.cu"), os.path.join(_HERE, "toploc_pool.cu"),
                 os.path.join(_HERE, "toploc_rotary.cu"), os.path.join(_HERE, "toploc_logits.cu")]
SOURCES = PROOF_SOURCES + MODEL_SOURCES
PROOF_HEADERS = [os.path.join(_INCLUDE, "toploc.h"), os.path.join(_INCLUDE, "toploc_device.cuh"),
                 os.path.join(_HERE, "nearest_ratio.cuh")]
MODEL_HEADERS = [os.path.join(_INCLUDE, "toploc.h"), os.path.join(_INCLUDE, "toploc_model.h"),
                 os.path.join(_HERE, "model_common.cuh"), os.path.join(_HERE, "attention_common.cuh"),
                 os.path.join(_HERE, "attention_tc.cuh"), os.path.join(_HERE, "sm100.cuh")]
HEADERS = PROOF_HEADERS + MODEL_HEADERS
LIBRARY = os.path.join(_HERE, "libtoploc.so")


def _nvcc():
    for cand in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if cand and (os.path.sep not in cand or os.path.exists(cand)):
            return cand
    return "nvcc"


def _object(source, verbose, force):
    """The source's object file, compiled where it is older than the source or a header."""
    obj = os.path.join(_HERE, "build", os.path.basename(source)[:-3] + ".o")
    headers = MODEL_HEADERS if source in MODEL_SOURCES else PROOF_HEADERS
    newest = max(os.path.getmtime(p) for p in [source, os.path.abspath(__file__)] + headers)
    if not force and os.path.exists(obj) and os.path.getmtime(obj) >= newest:
        return obj
    tmp = obj + ".tmp%d" % os.getpid()
    cmd = [_nvcc(), "-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-lineinfo", "-std=c++17",
           "-c", "-Xcompiler", "-fPIC", "-I", _INCLUDE]
    if verbose:
        cmd += ["-Xptxas", "-v"]
    subprocess.run(cmd + [source, "-o", tmp], check=True)
    os.replace(tmp, obj)
    return obj


def build(force=False, verbose=False):
    newest = max(os.path.getmtime(p) for p in SOURCES + HEADERS + [os.path.abspath(__file__)])
    if not force and os.path.exists(LIBRARY) and os.path.getmtime(LIBRARY) >= newest:
        return LIBRARY
    os.makedirs(os.path.join(_HERE, "build"), exist_ok=True)
    with ThreadPoolExecutor(len(SOURCES)) as pool:  # a compiler process per source
        objects = list(pool.map(lambda source: _object(source, verbose, force), SOURCES))
    tmp = LIBRARY + ".tmp%d" % os.getpid()
    subprocess.run([_nvcc(), "-gencode", "arch=compute_100a,code=sm_100a", "-shared", "-Xcompiler", "-fPIC"] +
                   objects + ["-o", tmp], check=True)
    os.replace(tmp, LIBRARY)
    return LIBRARY


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="--verbose" in sys.argv))
