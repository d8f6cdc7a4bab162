"""How long the pieces of an attention call for trees of new tokens are: the library's own rules, compiled for the host, applied to the lengths."""
import collections
import ctypes
import os
import subprocess

import common_prefix_plan as P

Plan = collections.namedtuple("Plan", "slots row_waves row_tiles ranges keys own_row_waves shares one_launch")
Own = collections.namedtuple("Own", "row_waves pieces tiles")     # tiles: of 32 keys, that a key group of a piece walks


def build(folder):
    out = str(folder / "libtree_walk.so")
    subprocess.run([os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "llvm", "bin", "clang++"), "-std=c++17", "-O1", "-fPIC", "-shared", "-Wno-ignored-attributes",
                    "-I" + os.path.join(P.HERE, "host_hip"), "-I" + P.CSRC, os.path.join(P.HERE, "host_hip", "tree_walk.cpp"), "-o", out], check=True)
    lib = ctypes.CDLL(out)
    lib.tree_walk_plan.argtypes = [ctypes.c_int64] * 2 + [ctypes.c_int] * 2 + [ctypes.c_int64] * 4 + [ctypes.c_void_p]
    lib.tree_walk_row_waves.argtypes = [ctypes.c_int64]
    return lib


def walks(lib, Hq, Hkv, prefix_len, lens, new, cus):
    """(plan, one Own a sequence) of a call whose bounds are what there is."""
    group, got = Hq // Hkv, (ctypes.c_int64 * 8)()
    assert lib.tree_walk_plan(sum(new), len(lens), Hq, Hkv, prefix_len, max(lens), max(new), cus, got)
    p = Plan(*got)
    parts, total = [], 0
    for L, n in zip(lens, new):
        rows, behind = n * group, max(L - prefix_len, 0) if n else 0
        w = min(lib.tree_walk_row_waves(rows), p.own_row_waves)
        steps = -(-behind // (32 * (4 // w)))
        total += steps * -(-rows // (32 * w)) * Hkv
        parts.append((w, steps))
    share = max(-(-total // max(p.shares, 1)), 1)
    own = []
    for w, steps in parts:
        pieces = -(-steps // share)
        if prefix_len == 0 and lib.tree_walk_one_piece(steps, share):
            pieces = min(pieces, 1)
        own.append(Own(w, pieces, -(-steps // pieces) if pieces else 0))
    return p, own
