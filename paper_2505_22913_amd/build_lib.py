"""Builds libmustafar.so (the gfx950 HIP kernels and their C ABI) in-tree.

    python -m paper_2505_22913_amd.build_lib          # build
    python -m paper_2505_22913_amd.build_lib --asm    # also dump gfx950 assembly

hipcc cross-compiles for gfx950 without a GPU. Packed-FP32 instruction
selection is disabled for every kernel.
"""
from __future__ import annotations

import argparse
import concurrent.futures
import os
import shutil
import subprocess
import sys
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIB = os.path.join(HERE, "libmustafar.so")
SOURCES = ["api.hip", "compress.hip", "attention.hip", "attention_mfma.hip", "measure.hip", "paged_api.hip", "paged.hip",
           "paged_attn.hip"]
ARCH = "gfx950"
# Per source: k_paged_chunk runs two waves a SIMD, one at d = 256; left to itself the compiler gives every
# matrix product an AGPR result and copies the scores, which the vector units read, out of them.
EXTRA_FLAGS = {"paged_attn.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form=1"]}


def hipcc() -> str:
    path = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(path):
        raise RuntimeError("hipcc not found: cannot build libmustafar.so")
    return path


def common_flags() -> list[str]:
    return [f"--offload-arch={ARCH}", "-O3", "-std=c++17", "-fPIC", "-Wall", "-fno-strict-aliasing",
            "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
            f"-I{INCLUDE}", f"-I{CSRC}"]


def build(verbose: bool = False) -> str:
    """Compiles every source to an object of its own, a few at a time, and links them."""
    def run(cmd):
        if verbose:
            print(" ".join(cmd), flush=True)
        subprocess.run(cmd, check=True)

    with tempfile.TemporaryDirectory() as objects:
        outs = [os.path.join(objects, s + ".o") for s in SOURCES]
        cmds = [[hipcc(), *common_flags(), *EXTRA_FLAGS.get(s, []), "-c", os.path.join(CSRC, s), "-o", o]
                for s, o in zip(SOURCES, outs)]
        with concurrent.futures.ThreadPoolExecutor(max_workers=4) as pool:
            list(pool.map(run, cmds))
        tmp = LIB + ".tmp"
        run([hipcc(), f"--offload-arch={ARCH}", "-shared", "-fPIC", "-o", tmp, *outs])
    os.replace(tmp, LIB)
    return LIB


def dump_asm(out_dir: str) -> None:
    """Device assembly of every source, for reading the generated gfx950 code."""
    os.makedirs(out_dir, exist_ok=True)
    for s in SOURCES:
        out = os.path.join(out_dir, s.replace(".hip", f"-{ARCH}.s"))
        cmd = [hipcc(), *common_flags(), *EXTRA_FLAGS.get(s, []), "--cuda-device-only", "-S", "-o", out,
               os.path.join(CSRC, s)]
        subprocess.run(cmd, check=True)


def main(argv=None) -> int:
    ap = argparse.ArgumentParser()
    ap.add_argument("--asm", metavar="DIR", help="write gfx950 assembly into DIR")
    ap.add_argument("-v", "--verbose", action="store_true")
    args = ap.parse_args(argv)
    print(build(verbose=args.verbose))
    if args.asm:
        dump_asm(args.asm)
    return 0


if __name__ == "__main__":
    sys.exit(main())
