"""Builds libahstage.so (HIP, gfx950 only) in-tree with hipcc."""
import concurrent.futures
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
OBJ = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libahstage.so")
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Xclang", "-target-feature", "-Xclang",
         "-packed-fp32-ops", "-I" + CSRC, "-I" + os.path.join(os.path.dirname(HERE), "include")]


# Per-file additions.  attention.hip: its softmax never produces a NaN (the running maximum is finite once the first
# key tile is seen, and every query sees key 0), so the compiler need not quiet possible signalling NaNs before every
# maximum (a third of the vector instructions behind the row maximum otherwise); infinities (the mask) stay honoured.
# And its kernels of more than 256 registers compute on their score tiles between matrix products: results of those
# products go to the ordinary registers, not to the accumulation registers from which every element would have to be
# copied (backward at 1 x 16 x 2048 x 128: 99 -> 91 us).  attention_window.hip: the same maxima (a query sees itself; a
# NaN in the inputs passes them by and shows through the exponentials); its dK/dV kernel of
# 128-wide heads is better off with the sums of dK and dV in the accumulation registers (4096 x 32 x 128, window 1024: 313 -> 299 us).
EXTRA = {"attention.hip": ["-fno-honor-nans", "-mllvm", "-amdgpu-mfma-vgpr-form=1"], "attention_window.hip": ["-fno-honor-nans"]}


def _compile(src):
    obj = os.path.join(OBJ, os.path.basename(src) + ".o")
    r = subprocess.run(["hipcc", *FLAGS, *EXTRA.get(os.path.basename(src), []), "-c", src, "-o", obj], capture_output=True, text=True)
    err = "\n".join(l for l in r.stderr.splitlines() if "packed-fp32-ops" not in l)
    if r.returncode != 0:
        raise RuntimeError("hipcc failed on %s:\n%s" % (src, err))
    return obj, err


def build(verbose=False):
    os.makedirs(OBJ, exist_ok=True)
    srcs = sorted(os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".hip"))
    with concurrent.futures.ThreadPoolExecutor(max_workers=min(8, len(srcs))) as ex:
        results = list(ex.map(_compile, srcs))
    for _, err in results:
        if verbose and err.strip():
            print(err, file=sys.stderr)
    r = subprocess.run(["hipcc", "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB, *[o for o, _ in results]],
                       capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("link failed:\n" + r.stderr)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
