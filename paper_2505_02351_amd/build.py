"""Builds liboptgqa.so (HIP kernels + C ABI) for gfx950, in-tree, with hipcc.

    python -m paper_2505_02351_amd.build            # compile
    python -m paper_2505_02351_amd.build --asm      # also keep the device assembly in _build/

The build needs no GPU (hipcc cross-compiles).  Packed-fp32 instruction selection is
switched off for all device code.
"""
from __future__ import annotations

import os
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
SRC = os.path.join(PKG, "csrc", "liboptgqa.hip")          # all of it in one file
PARTS = ("optgqa.hip", "operators.hip", "pages.hip")      # what SRC includes, compiled side by side
LIB = os.path.join(PKG, "liboptgqa.so")
BUILD_DIR = os.path.join(ROOT, "_build")

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wno-unused-command-line-argument", "-Werror=inline-asm",
]


def build(keep_asm: bool = False, verbose: bool = False, defines=(), out: str = LIB) -> str:
    """Compile csrc/*.hip.  `defines` (e.g. ["OPTGQA_RING_TILES=4"]) and `out` exist for
    tuning experiments; the product library is the default call."""
    os.makedirs(BUILD_DIR, exist_ok=True)
    tmp = os.path.join(BUILD_DIR, f"liboptgqa.{os.getpid()}.so")
    objects = [os.path.join(BUILD_DIR, f"{os.path.splitext(p)[0]}.{os.getpid()}.o") for p in PARTS]
    flags = [f for f in HIPCC_FLAGS if f != "-shared"]
    cmds = [["hipcc", *flags, "-c", *["-D" + d for d in defines], "-I" + os.path.join(ROOT, "include"), "-I" + os.path.join(PKG, "csrc"),
             *(["-save-temps=obj"] if keep_asm else []), os.path.join(PKG, "csrc", p), "-o", o] for p, o in zip(PARTS, objects)]
    try:
        running = [subprocess.Popen(c, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, cwd=BUILD_DIR) for c in cmds]
        said = [r.communicate()[0] for r in running]             # (all are waited for before any is judged)
        for r, text in zip(running, said):
            _judge(r.returncode, text, verbose)
        res = subprocess.run(["hipcc", *HIPCC_FLAGS, *objects, "-o", tmp], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, cwd=BUILD_DIR)
        _judge(res.returncode, res.stdout, verbose)
    finally:
        for o in objects:
            if os.path.exists(o):
                os.remove(o)
    os.replace(tmp, out)
    return out


def _judge(status: int, text: str, verbose: bool) -> None:
    noise = "'-packed-fp32-ops' is not a recognized feature"       # host pass does not know the feature
    err = "\n".join(l for l in text.splitlines() if noise not in l)
    if status != 0:
        raise RuntimeError(f"hipcc failed ({status}):\n{err}")
    if verbose and err.strip():
        print(err, file=sys.stderr)


if __name__ == "__main__":
    print(build(keep_asm="--asm" in sys.argv, verbose=True))
