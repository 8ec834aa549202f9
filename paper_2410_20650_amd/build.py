"""Builds libneuzip.so (HIP, gfx950 only) in-tree with hipcc."""
import os
import subprocess
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
# NEUZIP_LIBRARY points the binding at another build of the library (tuning runs); build() always writes the in-tree one
LIB = os.environ.get("NEUZIP_LIBRARY") or os.path.join(HERE, "libneuzip.so")
BUILT_LIB = os.path.join(HERE, "libneuzip.so")
# (the codec's translation unit first: it is the one whose kernels' metadata the tests read)
SOURCES = [os.path.join(HERE, "csrc", name) for name in ("neuzip.hip", "neuzip_embedding.hip", "neuzip_gated.hip", "neuzip_adapters.hip",
                                                   "neuzip_norm.hip", "neuzip_cache.hip", "neuzip_logits.hip")]
HEADERS = [os.path.join(ROOT, "include", "neuzip.h")] + [
    os.path.join(HERE, "csrc", name)
    for name in ("neuzip_format.h", "neuzip_host.h", "neuzip_walk.h", "neuzip_compress_kernels.h", "neuzip_decode_kernels.h",
                 "neuzip_linear_kernels.h", "neuzip_linear_launch.h", "neuzip_embedding_kernels.h",
                 "neuzip_gated_shape.h", "neuzip_gated_kernels.h", "neuzip_adapters_kernels.h", "neuzip_norm_kernels.h",
                 "neuzip_sequences.h", "neuzip_cache_kernels.h", "neuzip_attention_shape.h", "neuzip_attention_kernels.h", "neuzip_logits_kernels.h")]

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    "-Wall", "-Wno-unused-result",
    "-Wno-cuda-compat",  # (kernels in headers that two translation units include are inline)
    # packed fp32 instructions stay off for every HIP translation unit of this project
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
]


def is_stale() -> bool:
    if not os.path.exists(BUILT_LIB):
        return True
    built = os.path.getmtime(BUILT_LIB)
    return any(os.path.getmtime(p) > built for p in SOURCES + HEADERS)


def build(verbose: bool = False) -> str:
    """Compiles the translation units side by side and links them."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    with tempfile.TemporaryDirectory(prefix="neuzip_build_") as space:
        objects = [os.path.join(space, os.path.basename(source) + ".o") for source in SOURCES]
        running = []
        for source, made in zip(SOURCES, objects):
            cmd = [hipcc, *HIPCC_FLAGS, "-I", os.path.join(ROOT, "include"), "-c", source, "-o", made]
            if verbose:
                print(" ".join(cmd), flush=True)
            running.append((cmd, subprocess.Popen(cmd)))
        for cmd, process in running:
            if process.wait() != 0:
                for _, other in running:
                    other.kill()
                    other.wait()
                raise subprocess.CalledProcessError(process.returncode, cmd)
        cmd = [hipcc, "--offload-arch=gfx950", "-fPIC", "-shared", *objects, "-o", BUILT_LIB]
        if verbose:
            print(" ".join(cmd), flush=True)
        subprocess.run(cmd, check=True)
    return BUILT_LIB


if __name__ == "__main__":
    build(verbose=True)
