"""The library's own rules for cutting an attention call with one common prefix into pieces, compiled for the host."""
import collections
import ctypes
import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2505_02351_amd", "csrc")
Plan = collections.namedtuple("Plan", "row_waves row_tiles ranges keys own_row_waves shares pieces held")


def build(folder):
    """The rules as a shared library in `folder`."""
    out = str(folder / "libcommon_prefix.so")
    subprocess.run([os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "llvm", "bin", "clang++"), "-std=c++17", "-O1", "-fPIC", "-shared", "-Wno-ignored-attributes",
                    "-I" + os.path.join(HERE, "host_hip"), "-I" + CSRC, os.path.join(HERE, "host_hip", "common_prefix.cpp"), "-o", out], check=True)
    lib = ctypes.CDLL(out)
    lib.common_plan_of.argtypes = [ctypes.c_int64] * 2 + [ctypes.c_int] * 2 + [ctypes.c_int64] * 4 + [ctypes.c_void_p]
    return lib


def plan(lib, tokens, seqs, heads, kv_heads, prefix_len, max_context_len, max_q_len, cus=256):
    """The plan of a call, or None: refused."""
    out = (ctypes.c_int64 * 8)()
    return Plan(*out) if lib.common_plan_of(tokens, seqs, heads, kv_heads, prefix_len, max_context_len, max_q_len, cus, out) else None
