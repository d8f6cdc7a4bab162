"""Binding of the calls that stand around the attention of a step: rotary positions, rotated cache appends, the
attention of a batch with a common prefix and of trees of new tokens, and the verification of drafted tokens.

Conventions as in the package: q [T, Hq, D], k and v [T, Hkv, D] with any token stride (dense in their
last two dims: slices of one projection's rows will do), caches [NB, Hkv, bs, D], positions [T] int32,
slot_mapping [T] int64, freqs [rotary_dim / 2] float64.  Every output is the caller's.
"""
from __future__ import annotations

import ctypes
from typing import Optional, Tuple

import torch

import paper_2505_02351_amd as _pkg

# scaling of rotary_frequencies
ROTARY_PLAIN, ROTARY_LINEAR, ROTARY_BASE, ROTARY_YARN, ROTARY_WAVELENGTH = range(5)


def declare(lib: ctypes.CDLL) -> None:
    """The signatures of this module's entry points."""
    vp, i32, i64, f32, f64 = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_float, ctypes.c_double
    for name, args in {
        "rotary_frequencies_host": [vp, vp, i32, f64, i32, f64, f64, f64, f64],
        "rotary_embedding": [vp] * 6 + [i32] * 6 + [f32, i32] + [i64] * 4 + [i32, vp],
        "rotary_and_cache": [vp] * 9 + [i32] * 6 + [f32, i32] + [i64] * 4 + [i32, vp],
        "rotary_and_cache_fp8": [vp] * 9 + [i32] * 6 + [f32, i32] + [i64] * 4 + [f32, f32, i32, vp],
        "rotary_and_cache_fp8_heads": [vp] * 9 + [i32] * 6 + [f32, i32] + [i64] * 4 + [vp, vp, i32, vp],
        "paged_attention_common": [vp] * 9 + [f32] + [i32] * 10 + [vp, ctypes.c_size_t, i32, vp],
        "paged_attention_common_fp8": [vp] * 9 + [f32] * 3 + [i32] * 10 + [vp, ctypes.c_size_t, i32, vp],
        "paged_attention_common_fp8_heads": [vp] * 9 + [f32, vp, vp] + [i32] * 10 + [vp, ctypes.c_size_t, i32, vp],
        "paged_attention_tree": [vp] * 11 + [f32] + [i32] * 11 + [vp, ctypes.c_size_t, i32, vp],
        "paged_attention_tree_fp8": [vp] * 11 + [f32] * 3 + [i32] * 11 + [vp, ctypes.c_size_t, i32, vp],
        "paged_attention_tree_fp8_heads": [vp] * 11 + [f32, vp, vp] + [i32] * 11 + [vp, ctypes.c_size_t, i32, vp],
        "tree_masks_host": [vp] * 3 + [i32] * 2,
        "verify_drafts": [vp] * 8 + [i32] * 3 + [i64, i64, vp, ctypes.c_size_t, i32, vp],
    }.items():
        f = getattr(lib, "optgqa_" + name)
        f.restype, f.argtypes = i32, args
    for name, n in (("common_prefix_workspace_bytes", 9), ("tree_workspace_bytes", 9), ("verify_drafts_workspace_bytes", 2)):
        f = getattr(lib, "optgqa_" + name)
        f.restype, f.argtypes = ctypes.c_size_t, [i32] * n


def rotary_frequencies(rotary_dim: int, base: float = 10000.0, scaling: int = ROTARY_PLAIN, factor: float = 1.0,
                       original_len: float = 0.0, a: Optional[float] = None, b: Optional[float] = None) -> Tuple[torch.Tensor, float]:
    """optgqa_rotary_frequencies_host -> (frequencies [rotary_dim / 2] float64 on the CPU, magnitude).  a, b default to
    32 and 1 turns (ROTARY_YARN), 1 and 4 (ROTARY_WAVELENGTH)."""
    yarn = scaling == ROTARY_YARN
    a, b = (32.0 if yarn else 1.0) if a is None else a, (1.0 if yarn else 4.0) if b is None else b
    freqs, magnitude = torch.empty(max(int(rotary_dim) // 2, 1), dtype=torch.float64), ctypes.c_float(0.0)
    rc = _pkg.load_library().optgqa_rotary_frequencies_host(freqs.data_ptr(), ctypes.addressof(magnitude), int(rotary_dim), float(base),
                                                            int(scaling), float(factor), float(original_len), float(a), float(b))
    _pkg._check(rc, "optgqa_rotary_frequencies_host")
    return freqs, magnitude.value


# The checks below run on every call, and a call for one token is bound by them: a tensor costs 0.2 us here.
def _refuse(t, name: str, dtype: torch.dtype, index: int) -> None:
    """Why _check_tensors does not take a tensor: its type first, then its place."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"optgqa: {name} must be a torch.Tensor")
    if t.dtype != dtype:
        raise TypeError(f"optgqa: {name} must be {dtype}, got {t.dtype}")
    if index < 0:
        raise ValueError("optgqa: tensors must live in GPU memory")
    raise ValueError(f"optgqa: {name} is on {t.device}, expected GPU {index}")


def _check_tensors(index: int, tensors) -> None:
    """(tensor, name, type) each: element type, and GPU `index`.  Types before places, as everywhere in the package."""
    wrong = None
    for x in tensors:
        t = x[0]
        if type(t) is not torch.Tensor and not isinstance(t, torch.Tensor) or t.dtype is not x[2]:
            _refuse(*x, index)
        if t.get_device() != index or index < 0:
            wrong = wrong or x
    if wrong:
        _refuse(*wrong, index)


def _dense(*tensors) -> None:
    for t, name in tensors:
        if not t.is_contiguous():
            raise ValueError(f"optgqa: {name} must be contiguous")


# (a private name, as for _stream)
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _here(index: int) -> None:
    if _current_device() != index:
        raise ValueError(f"optgqa: the tensors are on GPU {index}, which is not the current one")


def _rows(t: torch.Tensor, name: str, tokens: int, D: int) -> Tuple[int, int]:
    """(heads, token stride) of a [T, heads, D] tensor whose tokens' rows are dense."""
    shape = t.shape
    if len(shape) != 3 or shape[0] != tokens or shape[2] != D:
        raise ValueError(f"optgqa: {name} must be [{tokens}, heads, {D}], got {tuple(shape)}")
    H, stride = shape[1], t.stride()
    if tokens and H and (stride[2] != 1 or (H > 1 and stride[1] != D)):
        raise ValueError(f"optgqa: {name} must be dense in its last two dims")
    return H, stride[0] if tokens > 1 else H * D


def _positions(positions, freqs, tokens: int, D: int) -> int:
    """rotary_dim, after checks of what the angles are made of."""
    if positions.shape != (tokens,) or not positions.is_contiguous():
        raise ValueError(f"optgqa: positions must be a dense tensor of {tokens} values")
    shape = freqs.shape
    if len(shape) != 1 or not freqs.is_contiguous() or not 0 < 2 * shape[0] <= D:
        raise ValueError(f"optgqa: freqs must be a dense tensor of 1 to {D // 2} values")
    return 2 * shape[0]


def rotary_embedding(q_out: torch.Tensor, q: torch.Tensor, k_out: Optional[torch.Tensor], k: Optional[torch.Tensor],
                     positions: torch.Tensor, freqs: torch.Tensor, *, interleaved: bool = False, magnitude: float = 1.0,
                     backward: bool = False, stream=None) -> None:
    """optgqa_rotary_embedding: q (and k, or None) turned by their positions; outputs may be the inputs.  backward:
    the gradient with respect to them, given that of the turned rows."""
    lib = _pkg.load_library()
    if (k is None) != (k_out is None):
        raise ValueError("optgqa: k and k_out come together")
    code, dtype = _pkg._dtype_code(q), q.dtype
    tensors = (q, "q", dtype), (q_out, "q_out", dtype), (positions, "positions", torch.int32), (freqs, "freqs", torch.float64)
    _check_tensors(q.get_device(), tensors if k is None else (*tensors, (k, "k", dtype), (k_out, "k_out", dtype)))
    T, D = q.shape[0], q.shape[-1]
    Hq, qs = _rows(q, "q", T, D)
    Ho, qos = _rows(q_out, "q_out", T, D)
    Hkv = Hko = ks = kos = 0
    if k is not None:
        Hkv, ks = _rows(k, "k", T, D)
        Hko, kos = _rows(k_out, "k_out", T, D)
    if Ho != Hq or Hko != Hkv:
        raise ValueError("optgqa: shape mismatch between q, k and their outputs")
    rot = _positions(positions, freqs, T, D)
    rc = lib.optgqa_rotary_embedding(q_out.data_ptr(), q.data_ptr(), _pkg._ptr(k_out), _pkg._ptr(k), positions.data_ptr(), freqs.data_ptr(),
                                     T, Hq, Hkv, D, rot, interleaved, magnitude, backward, qos, qs, kos, ks, code, _pkg._stream(stream))
    if rc:
        _pkg._check(rc, "optgqa_rotary_embedding")


def _append(name, q_out, q, k, v, k_cache, v_cache, slot_mapping, positions, freqs, interleaved, magnitude, stream, kv8, scales) -> None:
    lib = _pkg.load_library()
    code, dtype = _pkg._dtype_code(q), q.dtype
    cache = torch.uint8 if kv8 else dtype
    _check_tensors(q.get_device(), ((q, "q", dtype), (q_out, "q_out", dtype), (k, "k", dtype), (v, "v", dtype), (k_cache, "k_cache", cache),
                                    (v_cache, "v_cache", cache), (positions, "positions", torch.int32),
                                    (slot_mapping, "slot_mapping", torch.int64), (freqs, "freqs", torch.float64)))
    T, D = q.shape[0], q.shape[-1]
    shape = k_cache.shape
    NB, Hkv, bs, Dk = shape
    Hq, qs = _rows(q, "q", T, D)
    Ho, qos = _rows(q_out, "q_out", T, D)
    Hk, ks = _rows(k, "k", T, D)
    Hv, vs = _rows(v, "v", T, D)
    if Dk != D or v_cache.shape != shape or Ho != Hq or Hk != Hkv or Hv != Hkv:
        raise ValueError("optgqa: shape mismatch between q, q_out, k, v and the caches")
    if slot_mapping.shape != (T,):
        raise ValueError(f"optgqa: slot_mapping must have {T} values")
    _dense((k_cache, "k_cache"), (v_cache, "v_cache"), (slot_mapping, "slot_mapping"))
    rot = _positions(positions, freqs, T, D)
    rc = getattr(lib, name)(q_out.data_ptr(), q.data_ptr(), k.data_ptr(), v.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(),
                            slot_mapping.data_ptr(), positions.data_ptr(), freqs.data_ptr(), T, Hq, Hkv, D, rot, interleaved,
                            magnitude, bs, qos, qs, ks, vs, *scales, code, _pkg._stream(stream))
    if rc:
        _pkg._check(rc, name)


def rotary_and_cache(q_out: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, k_cache: torch.Tensor,
                     v_cache: torch.Tensor, slot_mapping: torch.Tensor, positions: torch.Tensor, freqs: torch.Tensor, *,
                     interleaved: bool = False, magnitude: float = 1.0, stream=None) -> None:
    """optgqa_rotary_and_cache: q turned into q_out (may be q), k turned and v stored in the paged caches, one launch."""
    _append("optgqa_rotary_and_cache", q_out, q, k, v, k_cache, v_cache, slot_mapping, positions, freqs, interleaved, magnitude, stream,
            False, ())


def rotary_and_cache_fp8(q_out: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, k_cache: torch.Tensor,
                         v_cache: torch.Tensor, slot_mapping: torch.Tensor, positions: torch.Tensor, freqs: torch.Tensor,
                         k_scale: float, v_scale: float, *, interleaved: bool = False, magnitude: float = 1.0, stream=None) -> None:
    """optgqa_rotary_and_cache_fp8: the same into E4M3 caches (uint8 tensors), one scale per tensor."""
    _append("optgqa_rotary_and_cache_fp8", q_out, q, k, v, k_cache, v_cache, slot_mapping, positions, freqs, interleaved, magnitude, stream,
            True, (float(k_scale), float(v_scale)))


def rotary_and_cache_fp8_heads(q_out: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, k_cache: torch.Tensor,
                               v_cache: torch.Tensor, slot_mapping: torch.Tensor, positions: torch.Tensor, freqs: torch.Tensor,
                               k_scales: torch.Tensor, v_scales: torch.Tensor, *, interleaved: bool = False, magnitude: float = 1.0,
                               stream=None) -> None:
    """optgqa_rotary_and_cache_fp8_heads: the same with one scale pair per KV head (float32 device tensors [Hkv])."""
    _pkg._head_scales(q, k_cache, k_scales, v_scales)
    _append("optgqa_rotary_and_cache_fp8_heads", q_out, q, k, v, k_cache, v_cache, slot_mapping, positions, freqs, interleaved, magnitude,
            stream, True, (k_scales.data_ptr(), v_scales.data_ptr()))


def common_prefix_workspace_bytes(num_tokens: int, num_seqs: int, num_heads: int, num_kv_heads: int, head_dim: int, block_size: int,
                                  num_prefix_blocks: int, max_context_len: int, max_q_len: int = 1) -> int:
    """optgqa_common_prefix_workspace_bytes: sized for the largest of each argument, a workspace serves every call."""
    return int(_pkg.load_library().optgqa_common_prefix_workspace_bytes(num_tokens, num_seqs, num_heads, num_kv_heads, head_dim, block_size,
                                                                        num_prefix_blocks, max_context_len, max_q_len))


def _common(name, out, q, k_cache, v_cache, prefix_table, block_tables, context_lens, cu_q_lens, alibi_slopes, scale, max_context_len,
            max_q_len, workspace, stream, kv8, scales, tree=()) -> None:
    """tree: () or (tree_masks, positions or None)."""
    lib = _pkg.load_library()
    code, dtype = _pkg._dtype_code(q), q.dtype
    cache, i32 = torch.uint8 if kv8 else dtype, torch.int32
    index = q.get_device()
    more = () if cu_q_lens is None else ((cu_q_lens, "cu_q_lens", i32),)
    if alibi_slopes is not None:
        more += ((alibi_slopes, "alibi_slopes", torch.float32),)
    if tree:
        more += ((tree[0], "tree_masks", i32),) if tree[1] is None else ((tree[0], "tree_masks", i32), (tree[1], "positions", i32))
    _check_tensors(index, ((q, "q", dtype), (out, "out", dtype), (k_cache, "k_cache", cache), (v_cache, "v_cache", cache),
                           (prefix_table, "prefix_table", i32), (block_tables, "block_tables", i32), (context_lens, "context_lens", i32), *more))
    shape, tables = k_cache.shape, block_tables.shape
    T, Hq, D = q.shape
    NB, Hkv, bs, Dk = shape
    B = context_lens.shape[0]
    if (Dk != D or out.shape != q.shape or v_cache.shape != shape or len(prefix_table.shape) != 1 or len(tables) != 2 or tables[0] != B
            or (T != B if cu_q_lens is None else cu_q_lens.shape != (B + 1,)) or (alibi_slopes is not None and alibi_slopes.shape != (Hq,))):
        raise ValueError("optgqa: shape mismatch between q, out, the tables, lengths, slopes and the caches")
    _dense((out, "out"), (q, "q"), (k_cache, "k_cache"), (v_cache, "v_cache"), (prefix_table, "prefix_table"), (block_tables, "block_tables"),
           (context_lens, "context_lens"))
    if cu_q_lens is not None:
        _dense((cu_q_lens, "cu_q_lens"))
    if alibi_slopes is not None:
        _dense((alibi_slopes, "alibi_slopes"))
    masks = words = ()
    if tree:
        shape = tree[0].shape
        if len(shape) != 2 or shape[0] != T or (tree[1] is not None and tree[1].shape != (T,)):
            raise ValueError("optgqa: shape mismatch between q, tree_masks and positions")
        _dense(*((t, name) for t, name in zip(tree, ("tree_masks", "positions")) if t is not None))
        _here(index)
        masks, words = (tree[0].data_ptr(), _pkg._ptr(tree[1])), (shape[1],)
    ws_bytes = _pkg._workspace(workspace, q)
    rc = getattr(lib, name)(out.data_ptr(), q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(), prefix_table.data_ptr(),
                            block_tables.data_ptr(), context_lens.data_ptr(), _pkg._ptr(cu_q_lens), *masks, _pkg._ptr(alibi_slopes), scale, *scales,
                            *words, T, B, Hq, Hkv, D, bs, prefix_table.shape[0], tables[1], max_context_len, max_q_len,
                            _pkg._ptr(workspace), ws_bytes, code, _pkg._stream(stream))
    if rc:
        _pkg._check(rc, name)


def paged_attention_common(out: torch.Tensor, q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, prefix_table: torch.Tensor,
                           block_tables: torch.Tensor, context_lens: torch.Tensor, cu_q_lens: Optional[torch.Tensor],
                           alibi_slopes: Optional[torch.Tensor], scale: float, max_context_len: int, max_q_len: int = 1,
                           workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    """optgqa_paged_attention_common: attention of each sequence's new tokens over a prefix that all sequences have in common
    (prefix_table [blocks] int32) and their own blocks behind it; cu_q_lens None: one new token each."""
    _common("optgqa_paged_attention_common", out, q, k_cache, v_cache, prefix_table, block_tables, context_lens, cu_q_lens, alibi_slopes,
            scale, max_context_len, max_q_len, workspace, stream, False, ())


def paged_attention_common_fp8(out: torch.Tensor, q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, prefix_table: torch.Tensor,
                               block_tables: torch.Tensor, context_lens: torch.Tensor, cu_q_lens: Optional[torch.Tensor],
                               alibi_slopes: Optional[torch.Tensor], scale: float, k_scale: float, v_scale: float, max_context_len: int,
                               max_q_len: int = 1, workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    """optgqa_paged_attention_common_fp8: the same over E4M3 caches (uint8 tensors), one scale per tensor."""
    _common("optgqa_paged_attention_common_fp8", out, q, k_cache, v_cache, prefix_table, block_tables, context_lens, cu_q_lens, alibi_slopes,
            scale, max_context_len, max_q_len, workspace, stream, True, (float(k_scale), float(v_scale)))


def paged_attention_common_fp8_heads(out: torch.Tensor, q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor,
                                     prefix_table: torch.Tensor, block_tables: torch.Tensor, context_lens: torch.Tensor,
                                     cu_q_lens: Optional[torch.Tensor], alibi_slopes: Optional[torch.Tensor], scale: float,
                                     k_scales: torch.Tensor, v_scales: torch.Tensor, max_context_len: int, max_q_len: int = 1,
                                     workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    """optgqa_paged_attention_common_fp8_heads: the same with one scale pair per KV head (float32 device tensors [Hkv])."""
    _pkg._head_scales(q, k_cache, k_scales, v_scales)
    _common("optgqa_paged_attention_common_fp8_heads", out, q, k_cache, v_cache, prefix_table, block_tables, context_lens, cu_q_lens,
            alibi_slopes, scale, max_context_len, max_q_len, workspace, stream, True, (k_scales.data_ptr(), v_scales.data_ptr()))


def tree_workspace_bytes(num_tokens: int, num_seqs: int, num_heads: int, num_kv_heads: int, head_dim: int, block_size: int,
                         num_prefix_blocks: int, max_context_len: int, max_q_len: int) -> int:
    """optgqa_tree_workspace_bytes: sized for the largest of each argument, a workspace serves every call."""
    return int(_pkg.load_library().optgqa_tree_workspace_bytes(num_tokens, num_seqs, num_heads, num_kv_heads, head_dim, block_size,
                                                               num_prefix_blocks, max_context_len, max_q_len))


def tree_masks(parents, mask_words: Optional[int] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """optgqa_tree_masks_host -> (masks [n, mask_words] int32, depths [n] int32) on the CPU, of a tree of n nodes: parents[i] < i, negative
    for a root.  mask_words: as many as n bits take, unless given."""
    parents = torch.as_tensor(parents, dtype=torch.int32, device="cpu").contiguous()
    if len(parents.shape) != 1:
        raise ValueError("optgqa: parents must have one dimension")
    n = parents.shape[0]
    words = max((n + 31) // 32, 1) if mask_words is None else int(mask_words)
    masks, depths = torch.zeros(n, max(words, 0), dtype=torch.int32), torch.zeros(n, dtype=torch.int32)
    _pkg._check(_pkg.load_library().optgqa_tree_masks_host(masks.data_ptr(), depths.data_ptr(), parents.data_ptr(), n, words), "optgqa_tree_masks_host")
    return masks, depths


def paged_attention_tree(out: torch.Tensor, q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, prefix_table: torch.Tensor,
                         block_tables: torch.Tensor, context_lens: torch.Tensor, cu_q_lens: Optional[torch.Tensor], tree_masks: torch.Tensor,
                         positions: Optional[torch.Tensor], alibi_slopes: Optional[torch.Tensor], scale: float, max_context_len: int,
                         max_q_len: int, workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    """optgqa_paged_attention_tree: paged_attention_common for trees of new tokens (prefix_table may be empty): each sees the keys
    before its sequence's new tokens, and of those the ones whose bits are set in its row of tree_masks [T, words] int32;
    positions [T] int32 (or None, without slopes): where they stand for the slopes."""
    _common("optgqa_paged_attention_tree", out, q, k_cache, v_cache, prefix_table, block_tables, context_lens, cu_q_lens, alibi_slopes,
            scale, max_context_len, max_q_len, workspace, stream, False, (), (tree_masks, positions))


def paged_attention_tree_fp8(out: torch.Tensor, q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, prefix_table: torch.Tensor,
                             block_tables: torch.Tensor, context_lens: torch.Tensor, cu_q_lens: Optional[torch.Tensor],
                             tree_masks: torch.Tensor, positions: Optional[torch.Tensor], alibi_slopes: Optional[torch.Tensor], scale: float,
                             k_scale: float, v_scale: float, max_context_len: int, max_q_len: int, workspace: Optional[torch.Tensor] = None,
                             stream=None) -> None:
    """optgqa_paged_attention_tree_fp8: the same over E4M3 caches (uint8 tensors), one scale per tensor."""
    _common("optgqa_paged_attention_tree_fp8", out, q, k_cache, v_cache, prefix_table, block_tables, context_lens, cu_q_lens, alibi_slopes,
            scale, max_context_len, max_q_len, workspace, stream, True, (float(k_scale), float(v_scale)), (tree_masks, positions))


def paged_attention_tree_fp8_heads(out: torch.Tensor, q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor,
                                   prefix_table: torch.Tensor, block_tables: torch.Tensor, context_lens: torch.Tensor,
                                   cu_q_lens: Optional[torch.Tensor], tree_masks: torch.Tensor, positions: Optional[torch.Tensor],
                                   alibi_slopes: Optional[torch.Tensor], scale: float, k_scales: torch.Tensor, v_scales: torch.Tensor,
                                   max_context_len: int, max_q_len: int, workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    """optgqa_paged_attention_tree_fp8_heads: the same with one scale pair per KV head (float32 device tensors [Hkv])."""
    _pkg._head_scales(q, k_cache, k_scales, v_scales)
    _common("optgqa_paged_attention_tree_fp8_heads", out, q, k_cache, v_cache, prefix_table, block_tables, context_lens, cu_q_lens,
            alibi_slopes, scale, max_context_len, max_q_len, workspace, stream, True, (k_scales.data_ptr(), v_scales.data_ptr()),
            (tree_masks, positions))


_PROBABILITIES = {torch.float16: _pkg.F16, torch.bfloat16: _pkg.BF16, torch.float32: 2}


def verify_drafts_workspace_bytes(num_seqs: int, vocab_size: int) -> int:
    """optgqa_verify_drafts_workspace_bytes."""
    return int(_pkg.load_library().optgqa_verify_drafts_workspace_bytes(num_seqs, vocab_size))


def verify_drafts(tokens: torch.Tensor, num_accepted: torch.Tensor, target_probs: torch.Tensor, draft_probs: Optional[torch.Tensor],
                  draft_tokens: torch.Tensor, cu_draft_lens: torch.Tensor, accept_uniforms: torch.Tensor, sample_uniforms: torch.Tensor,
                  workspace: Optional[torch.Tensor], stream=None) -> None:
    """optgqa_verify_drafts: which of the drafts are kept, and each sequence's next token.  tokens [B, max_drafts + 1] int64,
    target_probs [drafts + B, V] and draft_probs [drafts, V] (or None: drafts were certain) float32, float16 or bfloat16."""
    lib = _pkg.load_library()
    code = _PROBABILITIES.get(target_probs.dtype)
    if code is None:
        raise TypeError(f"optgqa: probabilities must be float32, float16 or bfloat16, got {target_probs.dtype}")
    index, i64, i32, f32 = target_probs.get_device(), torch.int64, torch.int32, torch.float32
    draft = () if draft_probs is None else ((draft_probs, "draft_probs", target_probs.dtype),)
    _check_tensors(index, (*draft, (tokens, "tokens", i64), (num_accepted, "num_accepted", i32), (draft_tokens, "draft_tokens", i64),
                           (cu_draft_lens, "cu_draft_lens", i32), (accept_uniforms, "accept_uniforms", f32), (sample_uniforms, "sample_uniforms", f32)))
    _dense((tokens, "tokens"), (num_accepted, "num_accepted"), (draft_tokens, "draft_tokens"), (cu_draft_lens, "cu_draft_lens"),
           (accept_uniforms, "accept_uniforms"), (sample_uniforms, "sample_uniforms"))
    B, T, wide, rows = num_accepted.shape[0], draft_tokens.shape[0], tokens.shape, target_probs.shape
    if len(rows) != 2 or len(wide) != 2:
        raise ValueError("optgqa: tokens and target_probs must have two dimensions")
    V = rows[1]
    if (wide[0] != B or wide[1] < 1 or rows[0] != T + B or cu_draft_lens.shape != (B + 1,) or accept_uniforms.shape != (T,)
            or sample_uniforms.shape != (B,) or (draft_probs is not None and draft_probs.shape != (T, V))):
        raise ValueError("optgqa: shape mismatch between the tokens, probabilities, drafts and random numbers")
    target_stride, draft_stride = _row_stride(target_probs, "target_probs"), 0 if draft_probs is None else _row_stride(draft_probs, "draft_probs")
    ws_bytes = _pkg._workspace(workspace, target_probs)
    rc = lib.optgqa_verify_drafts(tokens.data_ptr(), num_accepted.data_ptr(), target_probs.data_ptr(), _pkg._ptr(draft_probs),
                                  draft_tokens.data_ptr(), cu_draft_lens.data_ptr(), accept_uniforms.data_ptr(), sample_uniforms.data_ptr(),
                                  B, V, wide[1] - 1, target_stride, draft_stride, _pkg._ptr(workspace), ws_bytes, code, _pkg._stream(stream))
    if rc:
        _pkg._check(rc, "optgqa_verify_drafts")


def _row_stride(t: torch.Tensor, name: str) -> int:
    stride, shape = t.stride(), t.shape
    if shape[0] and shape[1] > 1 and stride[1] != 1:
        raise ValueError(f"optgqa: {name} must have dense rows")
    return stride[0] if shape[0] > 1 else shape[1]
