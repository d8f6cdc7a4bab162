"""Binding of the calls that change what the caches' pages hold and who holds them: sequences that fork, grow, shrink and end, a
pool that is compacted, blocks that are copied, accepted branches that move to the front.

A pool is block_tables [B, MB] int32, context_lens [B] int32 and ref_counts [NB] int32 (how many table entries in use hold a
block).  All of it stays on the GPU; caches of all layers are handed over as a CacheSet.
"""
from __future__ import annotations

import ctypes
from typing import List, Optional, Sequence, Tuple

import torch

import paper_2505_02351_amd as _pkg

from .operators import _check_tensors, _dense, _here


def declare(lib: ctypes.CDLL) -> None:
    """The signatures of this module's entry points."""
    vp, i32, size = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t
    for name, result, args in (
        ("resize_workspace_bytes", size, [i32] * 3),
        ("resize_sequences", i32, [vp] * 8 + [i32] * 6 + [vp, size, vp]),
        ("fork_sequences", i32, [vp] * 6 + [i32] * 5 + [vp]),
        ("compact_workspace_bytes", size, [i32]),
        ("compact_blocks", i32, [vp] * 5 + [i32] * 5 + [vp, size, vp]),
        ("copy_blocks", i32, [vp, i32, vp, vp, i32, i32, size, vp]),
        ("keep_tokens", i32, [vp, i32] + [vp] * 4 + [i32] * 8 + [vp]),
    ):
        f = getattr(lib, "optgqa_" + name)
        f.restype, f.argtypes = result, args


def _places(addresses: Sequence[int], size: int) -> List[int]:
    """The addresses of caches of `size` bytes, each once: a cache is worked on by the threads of one address, and those of
    another would move rows of it under their hands."""
    once = list(dict.fromkeys(addresses))
    low = sorted(once)
    if any(b - a < size for a, b in zip(low, low[1:])):
        raise ValueError("optgqa: caches must not overlap in part")
    return once


class CacheSet:
    """K and V caches of all layers ([NB, Hkv, bs, D] each, all alike), and their addresses on the GPU: made once, where the
    caches are (not under graph capture), and kept as long as they are.  One that several layers share may be there several
    times and counts once; others must not overlap."""

    def __init__(self, caches: Sequence[torch.Tensor]):
        self.caches: Tuple[torch.Tensor, ...] = tuple(caches)
        if not self.caches:
            raise ValueError("optgqa: a CacheSet needs at least one cache")
        for i, t in enumerate(self.caches):
            if not isinstance(t, torch.Tensor):
                raise TypeError(f"optgqa: cache {i} must be a torch.Tensor")
            if t.dtype not in (torch.float16, torch.bfloat16, torch.uint8) or t.dtype != self.caches[0].dtype:
                raise TypeError(f"optgqa: caches must be float16, bfloat16 or uint8, all alike, got {t.dtype} for cache {i}")
        first = self.caches[0]
        for i, t in enumerate(self.caches):
            if t.dim() != 4 or t.shape != first.shape or not t.is_contiguous():
                raise ValueError(f"optgqa: caches must be contiguous [NB, Hkv, bs, D] tensors, all alike, got {tuple(t.shape)} for cache {i}")
            if not t.is_cuda or t.get_device() != first.get_device():
                raise ValueError("optgqa: caches must live in the memory of one GPU")
            if t.data_ptr() % 16:
                raise ValueError(f"optgqa: cache {i} must lie on 16 bytes")
        self.shape, self.element_bytes, self.index = first.shape, first.element_size(), first.get_device()
        places = _places([t.data_ptr() for t in self.caches], first.numel() * first.element_size())
        self.pointers = torch.tensor(places, dtype=torch.int64, device=first.device)
        self.count = len(places)                                 # (of addresses: what the kernels go by)


def _cache_set(caches) -> CacheSet:
    if not isinstance(caches, CacheSet):
        raise TypeError(f"optgqa: caches must be a CacheSet, got {type(caches).__name__}")
    return caches


def _pool(block_tables, context_lens, ref_counts):
    """(rows, entries of a row, blocks) of a pool."""
    shape = block_tables.shape
    if len(shape) != 2 or context_lens.shape != (shape[0],) or len(ref_counts.shape) != 1:
        raise ValueError("optgqa: shape mismatch between block_tables, context_lens and ref_counts")
    return shape[0], shape[1], ref_counts.shape[0]


def resize_workspace_bytes(num_seqs: int, max_blocks_per_seq: int, num_blocks: int) -> int:
    """optgqa_resize_workspace_bytes."""
    return int(_pkg.load_library().optgqa_resize_workspace_bytes(num_seqs, max_blocks_per_seq, num_blocks))


def resize_sequences(block_tables: torch.Tensor, context_lens: torch.Tensor, ref_counts: torch.Tensor, new_lens: torch.Tensor,
                     slot_mapping: Optional[torch.Tensor], cu_new_lens: Optional[torch.Tensor], copies: torch.Tensor, counts: torch.Tensor,
                     block_size: int, max_change: int, workspace: Optional[torch.Tensor], stream=None) -> None:
    """optgqa_resize_sequences: sequences get their new lengths (0: they end), in place.  slot_mapping [tokens] int64 (or None):
    where the new tokens go; copies [B, 2]: blocks to copy first; counts [2]: how many, and blocks that were lacking."""
    lib, i32 = _pkg.load_library(), torch.int32
    index = block_tables.get_device()
    more = () if slot_mapping is None else ((slot_mapping, "slot_mapping", torch.int64), (cu_new_lens, "cu_new_lens", i32))
    _check_tensors(index, ((block_tables, "block_tables", i32), (context_lens, "context_lens", i32), (ref_counts, "ref_counts", i32),
                           (new_lens, "new_lens", i32), (copies, "copies", i32), (counts, "counts", i32), *more))
    B, MB, NB = _pool(block_tables, context_lens, ref_counts)
    if new_lens.shape != (B,) or copies.shape != (B, 2) or counts.shape != (2,) or (slot_mapping is not None and (
            len(slot_mapping.shape) != 1 or cu_new_lens.shape != (B + 1,))):
        raise ValueError("optgqa: shape mismatch between the pool, new_lens, slot_mapping, cu_new_lens, copies and counts")
    _dense((block_tables, "block_tables"), (context_lens, "context_lens"), (ref_counts, "ref_counts"), (new_lens, "new_lens"), (copies, "copies"),
           (counts, "counts"), *(x[:2] for x in more))
    ws_bytes = _pkg._workspace(workspace, block_tables)
    _here(index)
    rc = lib.optgqa_resize_sequences(block_tables.data_ptr(), context_lens.data_ptr(), ref_counts.data_ptr(), new_lens.data_ptr(),
                                     _pkg._ptr(slot_mapping), None if slot_mapping is None else cu_new_lens.data_ptr(), copies.data_ptr(),
                                     counts.data_ptr(), B, MB, NB, block_size, 0 if slot_mapping is None else slot_mapping.shape[0], max_change,
                                     _pkg._ptr(workspace), ws_bytes, _pkg._stream(stream))
    if rc:
        _pkg._check(rc, "optgqa_resize_sequences")


def fork_sequences(tables_out: torch.Tensor, lens_out: torch.Tensor, block_tables: torch.Tensor, context_lens: torch.Tensor,
                   ref_counts: torch.Tensor, parents: torch.Tensor, block_size: int, stream=None) -> None:
    """optgqa_fork_sequences: row i of tables_out, lens_out becomes row parents[i] of the old tables, blocks shared; sequences that are
    nobody's parent are freed."""
    lib, i32 = _pkg.load_library(), torch.int32
    index = block_tables.get_device()
    _check_tensors(index, ((block_tables, "block_tables", i32), (context_lens, "context_lens", i32), (ref_counts, "ref_counts", i32),
                           (tables_out, "tables_out", i32), (lens_out, "lens_out", i32), (parents, "parents", i32)))
    B, MB, NB = _pool(block_tables, context_lens, ref_counts)
    N = lens_out.shape[0] if len(lens_out.shape) == 1 else -1
    if tables_out.shape != (N, MB) or parents.shape != (N,):
        raise ValueError("optgqa: shape mismatch between the old tables, the new ones and parents")
    _dense((block_tables, "block_tables"), (context_lens, "context_lens"), (ref_counts, "ref_counts"), (tables_out, "tables_out"),
           (lens_out, "lens_out"), (parents, "parents"))
    _here(index)
    rc = lib.optgqa_fork_sequences(tables_out.data_ptr(), lens_out.data_ptr(), block_tables.data_ptr(), context_lens.data_ptr(),
                                   ref_counts.data_ptr(), parents.data_ptr(), N, B, MB, NB, block_size, _pkg._stream(stream))
    if rc:
        _pkg._check(rc, "optgqa_fork_sequences")


def compact_workspace_bytes(num_blocks: int) -> int:
    """optgqa_compact_workspace_bytes."""
    return int(_pkg.load_library().optgqa_compact_workspace_bytes(num_blocks))


def compact_blocks(block_tables: torch.Tensor, context_lens: torch.Tensor, ref_counts: torch.Tensor, copies: torch.Tensor,
                   counts: torch.Tensor, block_size: int, workspace: Optional[torch.Tensor], stream=None) -> None:
    """optgqa_compact_blocks: the highest blocks in use go to the lowest free ones, at most copies.shape[0] of them; copies [.., 2]
    and counts [2] (pairs, blocks in use) are for copy_blocks, which has to follow."""
    lib, i32 = _pkg.load_library(), torch.int32
    index = block_tables.get_device()
    _check_tensors(index, ((block_tables, "block_tables", i32), (context_lens, "context_lens", i32), (ref_counts, "ref_counts", i32),
                           (copies, "copies", i32), (counts, "counts", i32)))
    B, MB, NB = _pool(block_tables, context_lens, ref_counts)
    if len(copies.shape) != 2 or copies.shape[1] != 2 or counts.shape != (2,):
        raise ValueError("optgqa: copies must be [pairs, 2] and counts [2]")
    _dense((block_tables, "block_tables"), (context_lens, "context_lens"), (ref_counts, "ref_counts"), (copies, "copies"), (counts, "counts"))
    ws_bytes = _pkg._workspace(workspace, block_tables)
    _here(index)
    rc = lib.optgqa_compact_blocks(block_tables.data_ptr(), context_lens.data_ptr(), ref_counts.data_ptr(), copies.data_ptr(), counts.data_ptr(),
                                   B, MB, NB, block_size, copies.shape[0], _pkg._ptr(workspace), ws_bytes, _pkg._stream(stream))
    if rc:
        _pkg._check(rc, "optgqa_compact_blocks")


def copy_blocks(caches: CacheSet, copies: torch.Tensor, num_copies: torch.Tensor, stream=None) -> None:
    """optgqa_copy_blocks: in all caches the blocks of the first num_copies[0] pairs (from, to) of copies are copied."""
    lib, i32 = _pkg.load_library(), torch.int32
    s = _cache_set(caches)
    _check_tensors(s.index, ((copies, "copies", i32), (num_copies, "num_copies", i32)))
    if len(copies.shape) != 2 or copies.shape[1] != 2 or len(num_copies.shape) != 1 or num_copies.shape[0] < 1:
        raise ValueError("optgqa: copies must be [pairs, 2] and num_copies [1] or more")
    _dense((copies, "copies"), (num_copies, "num_copies"))
    _here(s.index)
    NB, Hkv, bs, D = s.shape
    rc = lib.optgqa_copy_blocks(s.pointers.data_ptr(), s.count, copies.data_ptr(), num_copies.data_ptr(), copies.shape[0], NB,
                                Hkv * bs * D * s.element_bytes, _pkg._stream(stream))
    if rc:
        _pkg._check(rc, "optgqa_copy_blocks")


def keep_tokens(caches: CacheSet, block_tables: torch.Tensor, start_lens: torch.Tensor, paths: torch.Tensor, path_lens: torch.Tensor,
                stream=None) -> None:
    """optgqa_keep_tokens: in all caches row start_lens[b] + paths[b][i] of sequence b goes to row start_lens[b] + i, for i <
    path_lens[b]; paths [B, P] ascend."""
    lib, i32 = _pkg.load_library(), torch.int32
    s = _cache_set(caches)
    _check_tensors(s.index, ((block_tables, "block_tables", i32), (start_lens, "start_lens", i32), (paths, "paths", i32), (path_lens, "path_lens", i32)))
    tables, places = block_tables.shape, paths.shape
    if len(tables) != 2 or len(places) != 2 or places[0] != tables[0] or start_lens.shape != (tables[0],) or path_lens.shape != (tables[0],):
        raise ValueError("optgqa: shape mismatch between block_tables, start_lens, paths and path_lens")
    _dense((block_tables, "block_tables"), (start_lens, "start_lens"), (paths, "paths"), (path_lens, "path_lens"))
    _here(s.index)
    NB, Hkv, bs, D = s.shape
    rc = lib.optgqa_keep_tokens(s.pointers.data_ptr(), s.count, block_tables.data_ptr(), start_lens.data_ptr(), paths.data_ptr(),
                                path_lens.data_ptr(), tables[0], places[1], tables[1], NB, Hkv, D, bs, s.element_bytes, _pkg._stream(stream))
    if rc:
        _pkg._check(rc, "optgqa_keep_tokens")
