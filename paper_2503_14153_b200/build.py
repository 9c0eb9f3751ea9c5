"""Builds libspec_decode.so (sm_100a) next to the sources with nvcc."""
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libspec_decode.so")
_SHARED = ["common.cuh", os.path.join("..", "..", "include", "spec_decode.h")]
# each source file with the headers that it is built from, besides _SHARED
SOURCES = {
    "spec_api.cu": ["kernels_simple.cuh", "gemm_stream.cuh", "gemm_cluster.cuh", "gemm_glu.cuh", "gemm_pair.cuh", "glue_tc.cuh", "attention_tc.cuh",
                    "attention_umma.cuh", "labels.cuh"],
    "cache_api.cu": ["cache_common.cuh", "cache_rows.cuh", "cache_pages.cuh", "cache_attention.cuh", "cache_umma.cuh"],
}


def _newest(source: str) -> float:
    return max(os.path.getmtime(os.path.join(CSRC, d)) for d in [source] + SOURCES[source] + _SHARED if os.path.exists(os.path.join(CSRC, d)))


def _object(source: str) -> str:
    return os.path.join(HERE, "_build", os.path.splitext(source)[0] + ".o")


def needs_build() -> bool:
    return not os.path.exists(LIB) or any(_newest(s) > os.path.getmtime(LIB) for s in SOURCES)


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and not needs_build():
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    os.makedirs(os.path.join(HERE, "_build"), exist_ok=True)
    flags = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17", "-Xcompiler", "-fPIC", "-Xptxas", "-v" if verbose else "-O3"]
    jobs = [(s, subprocess.Popen([nvcc, *flags, "-c", "-o", _object(s), os.path.join(CSRC, s)], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True))
            for s in SOURCES if force or not os.path.exists(_object(s)) or _newest(s) > os.path.getmtime(_object(s))]
    failed = False
    for source, job in jobs:
        text = job.communicate()[0]
        if job.returncode != 0:
            sys.stderr.write(text)
            if os.path.exists(_object(source)):
                os.remove(_object(source))
            failed = True
        elif verbose:
            print(text)
    if failed:
        raise RuntimeError("nvcc failed")
    res = subprocess.run([nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-shared", "-cudart", "static", "-o", LIB] + [_object(s) for s in SOURCES],
                         capture_output=True, text=True)
    if res.returncode != 0:
        sys.stderr.write(res.stdout + res.stderr)
        raise RuntimeError("nvcc failed")
    return LIB


if __name__ == "__main__":
    print(build(force=True, verbose="-v" in sys.argv))
