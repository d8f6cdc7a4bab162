"""CPU: differences of positions, for any two of them."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

import common_prefix_plan as P


@pytest.fixture(scope="module")
def differences(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("distance") / "libdistance.so")
    subprocess.run([os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "llvm", "bin", "clang++"), "-std=c++17", "-O1", "-ffp-contract=off", "-fPIC", "-shared",
                    "-Wno-ignored-attributes", "-I" + os.path.join(P.HERE, "host_hip"), "-I" + P.CSRC, os.path.join(P.HERE, "host_hip", "distance.cpp"), "-o", out],
                   check=True)
    f = ctypes.CDLL(out).whole_differences
    f.argtypes = [ctypes.c_void_p] * 3 + [ctypes.c_int] * 2

    def run(a, b, less):
        a, b, got = np.array(a, np.int32), np.array(b, np.int32), np.zeros(len(a), np.float32)
        f(got.ctypes.data, a.ctypes.data, b.ctypes.data, less, len(a))
        return got, (a.astype(np.int64) - b.astype(np.int64) - less).astype(np.float32)        # (int64 to float32: one rounding)

    return run


@pytest.mark.parametrize("less", [0, 1, 27, 31])
def test_whole_differences(differences, less):
    edges = [v + d for v in (-2 ** 31, -2 ** 30, -2 ** 24, -2 ** 16, 0, 2 ** 16, 2 ** 24, 2 ** 30, 2 ** 31 - 1) for d in (-65537, -65536, -33, -2, -1, 0, 1, 2, 33, 65535, 65536)]
    edges = [v for v in edges if -2 ** 31 <= v < 2 ** 31]
    got, want = differences(np.repeat(edges, len(edges)), edges * len(edges), less)
    assert (got == want).all()
    rng = np.random.RandomState(less)
    for bits in (4, 12, 20, 31):
        a = rng.randint(-2 ** 31, 2 ** 31, 200000)
        b = np.clip(a + rng.randint(-2 ** bits, 2 ** bits, 200000), -2 ** 31, 2 ** 31 - 1) if bits < 31 else rng.randint(-2 ** 31, 2 ** 31, 200000)
        got, want = differences(a, b, less)
        assert (got == want).all()
