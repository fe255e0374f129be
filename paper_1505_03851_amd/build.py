"""Build the HIP libraries in-tree for gfx950: liblda_draw.so (the draw and
its C ABI, include/lda_draw.h) and liblda_probe.so (the measurement probes,
include/lda_probe.h)."""
from __future__ import annotations

import concurrent.futures
import os
import subprocess
import tempfile

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
# the draw library: its C ABI with the default build of the kernels, the build
# for tables past 4 GiB (lda_draw_wide.hip), the token operators, and the norm,
# the 8-bit product and the sampling
SRC = [os.path.join(PKG, "csrc", name)
       for name in ("lda_draw.hip", "lda_draw_wide.hip", "lda_tokens.hip", "lda_norm.hip",
                    "lda_product.hip", "lda_sample.hip")]
LIB = os.path.join(PKG, "liblda_draw.so")
PROBE_SRC = os.path.join(PKG, "csrc", "probe.hip")
PROBE_LIB = os.path.join(PKG, "liblda_probe.so")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

FLAGS = [
    "--offload-arch=gfx950",
    "-O3",
    "-std=c++17",
    "-fPIC",
    "-shared",
    # fp32 subnormals are kept (the products of small Dirichlet weights are
    # often subnormal); a*b+c may contract to one fused multiply-add.
    "-fno-gpu-flush-denormals-to-zero",
    "-ffp-contract=fast",
    # no packed-fp32 instructions in generated code
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall",
    "-I", os.path.join(ROOT, "include"),
]


def _run(cmd: list[str], verbose: bool) -> None:
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.run(cmd, check=True)


def _compile(src: str | list[str], lib: str, verbose: bool, extra: list[str] | None) -> str:
    srcs = [src] if isinstance(src, str) else list(src)
    flags = [*FLAGS, *(extra or [])]
    compiling = [f for f in flags if f != "-shared"]
    if len(srcs) == 1:
        _run([HIPCC, *flags, *srcs, "-o", lib + ".tmp"], verbose)
    else:  # the sources at once, then the library of what they gave
        with tempfile.TemporaryDirectory() as folder:
            objects = [os.path.join(folder, os.path.basename(s) + ".o") for s in srcs]
            with concurrent.futures.ThreadPoolExecutor(len(srcs)) as pool:
                jobs = [pool.submit(_run, [HIPCC, *compiling, "-c", s, "-o", o], verbose)
                        for s, o in zip(srcs, objects)]
                for job in jobs:
                    job.result()
            _run([HIPCC, *flags, *objects, "-o", lib + ".tmp"], verbose)
    os.replace(lib + ".tmp", lib)
    return lib


def build(verbose: bool = False, extra: list[str] | None = None) -> str:
    """Both libraries; returns the draw library's path."""
    _compile(PROBE_SRC, PROBE_LIB, verbose, extra)
    return _compile(SRC, LIB, verbose, extra)


if __name__ == "__main__":
    print(build(verbose=True))
