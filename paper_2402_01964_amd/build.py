"""Build ``libnlb.so`` (gfx950 kernels + the C ABI of include/nlb.h) in-tree."""
import os
import subprocess
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
SRCS = [os.path.join(HERE, "csrc", f) for f in (
    "nlb.hip", "aggregate.hip", "rnn.hip", "attention.hip", "attention_backward.hip", "layer_norm.hip")]
LIB = os.path.join(HERE, "libnlb.so")

HIPCC_FLAGS = [
    "-O3", "-std=c++17", "--offload-arch=gfx950", "-fPIC", "-shared",
    "-ffp-contract=off",
    # packed fp32 instructions are kept out of all device code
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    # matrix-core accumulators in ordinary VGPRs: the accumulate chains then
    # stay in place instead of being copied between register files
    "-mllvm", "-amdgpu-mfma-vgpr-form=1",
    "-Wall",
]


def build(verbose: bool = False) -> str:
    """Compile every source (side by side, eight at most) and link them."""
    hipcc = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "bin", "hipcc")

    def run(cmd):
        if verbose:
            print(" ".join(cmd), flush=True)
        subprocess.run(cmd, check=True)

    with tempfile.TemporaryDirectory() as d:
        objs = [os.path.join(d, os.path.basename(s) + ".o") for s in SRCS]
        flags = [f for f in HIPCC_FLAGS if f != "-shared"]
        with ThreadPoolExecutor(8) as pool:
            list(pool.map(lambda so: run([hipcc, *flags, "-I", os.path.join(ROOT, "include"), "-c", so[0], "-o",
                                          so[1]]), zip(SRCS, objs)))
        run([hipcc, "--offload-arch=gfx950", "-fPIC", "-shared", "-o", LIB + ".tmp", *objs])
    os.replace(LIB + ".tmp", LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
