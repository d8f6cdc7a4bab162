"""CPU: the slots that a resize gives to a sequence's new tokens never name a row outside of the pool."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

import common_prefix_plan as P


@pytest.fixture(scope="module")
def apply(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("pages") / "libpages.so")
    subprocess.run([os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "llvm", "bin", "clang++"), "-std=c++17", "-O1", "-fwrapv", "-fPIC", "-shared", "-Wno-ignored-attributes",
                    "-I" + os.path.join(P.HERE, "host_hip"), "-I" + P.CSRC, os.path.join(P.HERE, "host_hip", "pages.cpp"), "-o", out], check=True)
    f, vp, i32 = ctypes.CDLL(out).resize_apply_of, ctypes.c_void_p, ctypes.c_int
    f.restype, f.argtypes = None, [vp, vp, vp, i32, vp, vp] + [i32] * 6 + [vp, i32, i32]

    def run(row, old, new, last, fresh, cu, num_slots, num_blocks, bs=16, enough=True, step=1):
        """(row, length, slots): -2 where nothing was written."""
        length, refs = np.array([old], np.int32), np.zeros(num_blocks, np.int32)
        slots, cu, fresh = np.full(num_slots, -2, np.int64), np.array(cu, np.int32), np.array([*fresh, -9], np.int32)
        f(row.ctypes.data, length.ctypes.data, refs.ctypes.data, new, slots.ctypes.data, cu.ctypes.data, num_slots, row.shape[0], num_blocks,
          bs.bit_length() - 1, old, last, fresh.ctypes.data, int(enough), step)
        return row, int(length[0]), slots

    return run


@pytest.mark.parametrize("step", [1, 3])
@pytest.mark.parametrize("bad", [-1, -7, 30, 31, 1 << 28, 2 ** 31 - 1, -2 ** 31])
def test_tokens_of_a_last_block_that_is_none(apply, bad, step):
    """A row of 20 tokens whose second entry names no block grows to 37: tokens 20 .. 31 have no row, 32 .. 36 lie in its new block."""
    row, length, slots = apply(np.array([5, bad, -7, -7], np.int32), 20, 37, -1, [8], [0, 17], 19, 30, step=step)
    assert row.tolist() == [5, bad, 8, -7] and length == 37
    assert slots.tolist() == [-1] * 12 + [8 * 16 + i for i in range(5)] + [-2, -2]


def test_tokens_of_a_last_block_that_is_one(apply):
    assert apply(np.array([5, 29, -7], np.int32), 20, 37, -1, [8], [0, 18], 18, 30)[2].tolist() == [29 * 16 + i for i in range(4, 16)] + [128 + i for i in range(5)] + [-1]
    # replaced: held by others too
    row, _, slots = apply(np.array([5, 29, -7], np.int32), 20, 37, 29, [2, 8], [0, 17], 17, 30)
    assert row.tolist() == [5, 2, 8] and slots.tolist() == [2 * 16 + i for i in range(4, 16)] + [128 + i for i in range(5)]
    assert apply(np.array([5, 29, -7], np.int32), 20, 37, -1, [], [0, 17], 17, 30, enough=False)[1:][1].tolist() == [-1] * 17


def test_more_slots_than_tokens_at_the_longest_length(apply):
    """Places behind a sequence's new tokens are -1 also where a token there would have a position beyond 2^31."""
    bs, old, new = 16, 2 ** 31 - 20, 2 ** 31 - 2
    row = np.zeros(2 ** 27, np.int32)                        # (pages that nobody touches take no memory)
    row[-2] = 3
    slots = apply(row, old, new, -1, [7], [0, 60], 60, 30)[2]
    want = [3 * 16 + i for i in range(12, 16)] + [7 * 16 + i for i in range(14)]
    assert slots.tolist() == want + [-1] * (60 - len(want))


@pytest.mark.parametrize("cu", [[2 ** 31 - 1, -2 ** 31], [2 ** 31 - 1, -9], [-2 ** 31, -2 ** 31], [2 ** 31 - 1, 2 ** 31 - 1], [40, 2 ** 31 - 1], [19, 0]])
def test_prefix_sums_that_are_none_write_no_slot(apply, cu):
    """Room for 19 tokens, prefix sums outside of it."""
    assert (apply(np.array([5, 29, -7], np.int32), 20, 37, -1, [8], cu, 19, 30)[2] == -2).all()
