"""CPU: how a call for trees of new tokens is cut into pieces: the ranges cover the prefix, and what is held for a call holds it and
every call that is no larger in any of its sizes."""
import ctypes
import os
import random
import subprocess

import pytest

import common_prefix_plan as P

HEADS = [(32, 8), (32, 4), (64, 8), (8, 2), (40, 8), (16, 16), (8, 1), (5, 1), (48, 48), (512, 512)]


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("rules") / "libtree.so")
    subprocess.run([os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "llvm", "bin", "clang++"), "-std=c++17", "-O1", "-fPIC", "-shared", "-Wno-ignored-attributes",
                    "-I" + os.path.join(P.HERE, "host_hip"), "-I" + P.CSRC, os.path.join(P.HERE, "host_hip", "tree.cpp"), "-o", out], check=True)
    lib = ctypes.CDLL(out)
    lib.tree_plan_of.argtypes = [ctypes.c_int64] * 2 + [ctypes.c_int] * 2 + [ctypes.c_int64] * 4 + [ctypes.c_void_p]

    def of(*sizes):
        got = (ctypes.c_int64 * 5)()
        assert lib.tree_plan_of(*sizes, got), sizes
        return dict(zip(("tiles", "ranges", "keys", "pieces", "held"), got))

    return of


@pytest.mark.parametrize("cus", [256, 304, 32, 1])
def test_pieces_fit_and_smaller_calls_do(plan, cus):
    rng = random.Random(cus)

    def some(hi):
        return int(round(hi ** rng.random()))

    for _ in range(6000):
        Hq, Hkv = rng.choice(HEADS)
        new, B = some(100), some(200)
        prefix = 16 * rng.choice([0, some(20), some(2048)])
        most = prefix + rng.choice([0, some(300), some(40000)])
        tokens = rng.choice([B * new, some(B * new)])
        p = plan(tokens, B, Hq, Hkv, prefix, most, new, cus)
        assert 0 <= p["pieces"] <= p["held"], (tokens, B, Hq, Hkv, prefix, most, new)
        assert p["ranges"] * p["keys"] >= prefix and (prefix == 0 or (p["ranges"] - 1) * p["keys"] < prefix)
        for _ in range(3):
            b, n, shorter = rng.randint(1, B), rng.randint(1, new), 16 * rng.randint(0, prefix // 16)
            t, m = rng.randint(1, tokens), rng.randint(0, most)
            assert plan(t, b, Hq, Hkv, shorter, m, n, cus)["pieces"] <= p["held"], (tokens, B, Hq, Hkv, prefix, most, new, t, b, shorter, m, n)


def test_every_short_prefix_fits(plan):
    for Hq, Hkv in HEADS:
        for tokens in (1, 5, 33, 130, 700):
            for blocks in range(0, 40):
                p = plan(tokens, 5, Hq, Hkv, 16 * blocks, 16 * blocks, 200, 256)
                assert p["pieces"] <= p["held"], (Hq, Hkv, tokens, blocks)
