"""Binding of the calls that stand around the attention of a step: rotary positions, rotated cache appends, the
attention of a batch with a common prefix and the verification of drafted tokens.

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
        "verify_drafts": [vp] * 8 + [i32] * 3 + [i64, i64, vp, ctypes.c_size_t, i32, vp],
    }.items():
        f = getattr(lib, "optgqa_" + name)
        f.restype, f.argtypes = i32, args
    for name, n in (("common_prefix_workspace_bytes", 9), ("verify_drafts_workspace_bytes", 2)):
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


def _rows(t: torch.Tensor, name: str, tokens: int) -> Tuple[int, int]:
    """(heads, token stride) of a [T, heads, D] tensor whose tokens' rows are dense."""
    if t.dim() != 3 or t.shape[0] != tokens:
        raise ValueError(f"optgqa: {name} must be [{tokens}, heads, head_dim], got {tuple(t.shape)}")
    T, H, D = t.shape
    if T and H and (t.stride(2) != 1 or (H > 1 and t.stride(1) != D)):
        raise ValueError(f"optgqa: {name} must be dense in its last two dims")
    return H, t.stride(0) if T > 1 else H * D


def _positions(positions, freqs, tokens: int, D: int) -> int:
    """rotary_dim, after checks of what the angles are made of."""
    if positions.shape != (tokens,) or not positions.is_contiguous():
        raise ValueError(f"optgqa: positions must be a dense tensor of {tokens} values")
    if freqs.dim() != 1 or not freqs.is_contiguous() or not 0 < 2 * freqs.shape[0] <= D:
        raise ValueError(f"optgqa: freqs must be a dense tensor of 1 to {D // 2} values")
    return 2 * freqs.shape[0]


def rotary_embedding(q_out: torch.Tensor, q: torch.Tensor, k_out: Optional[torch.Tensor], k: Optional[torch.Tensor],
                     positions: torch.Tensor, freqs: torch.Tensor, *, interleaved: bool = False, magnitude: float = 1.0,
                     backward: bool = False, stream=None) -> None:
    """optgqa_rotary_embedding: q (and k, or None) turned by their positions; outputs may be the inputs.  backward:
    the gradient with respect to them, given that of the turned rows."""
    lib = _pkg.load_library()
    if (k is None) != (k_out is None):
        raise ValueError("optgqa: k and k_out come together")
    _pkg._typed(q, same=(("q_out", q_out), ("k", k), ("k_out", k_out)), i32=(("positions", positions),), f64=(("freqs", freqs),))
    T, D = q.shape[0], q.shape[-1]
    Hq, qs = _rows(q, "q", T)
    if q_out.shape != q.shape or (k is not None and (k_out.shape != k.shape or k.shape[-1] != D)):
        raise ValueError("optgqa: shape mismatch between q, k and their outputs")
    qos = _rows(q_out, "q_out", T)[1]
    Hkv, ks, kos = 0, 0, 0
    if k is not None:
        Hkv, ks = _rows(k, "k", T)
        kos = _rows(k_out, "k_out", T)[1]
    rot = _positions(positions, freqs, T, D)
    rc = lib.optgqa_rotary_embedding(q_out.data_ptr(), q.data_ptr(), _pkg._ptr(k_out), _pkg._ptr(k), positions.data_ptr(), freqs.data_ptr(),
                                     T, Hq, Hkv, D, rot, bool(interleaved), magnitude, bool(backward), qos, qs, kos, ks,
                                     _pkg._dtype_code(q), _pkg._stream(stream))
    _pkg._check(rc, "optgqa_rotary_embedding")


def _append(name, q_out, q, k, v, k_cache, v_cache, slot_mapping, positions, freqs, interleaved, magnitude, stream, kv8, scales) -> None:
    lib = _pkg.load_library()
    caches = (("k_cache", k_cache), ("v_cache", v_cache))
    rows = (("q_out", q_out), ("k", k), ("v", v))
    _pkg._typed(q, same=rows if kv8 else rows + caches, u8=caches if kv8 else (), i32=(("positions", positions),),
                i64=(("slot_mapping", slot_mapping),), f64=(("freqs", freqs),))
    T, D = q.shape[0], q.shape[-1]
    NB, Hkv, bs, Dk = k_cache.shape
    Hq, qs = _rows(q, "q", T)
    if Dk != D or v_cache.shape != k_cache.shape or q_out.shape != q.shape or k.shape[1:] != (Hkv, D) or v.shape[1:] != (Hkv, D):
        raise ValueError("optgqa: shape mismatch between q, q_out, k, v and the caches")
    if slot_mapping.shape != (T,):
        raise ValueError(f"optgqa: slot_mapping must have {T} values")
    for t, n in ((k_cache, "k_cache"), (v_cache, "v_cache"), (slot_mapping, "slot_mapping")):
        _pkg._dense(t, n)
    qos, ks, vs = _rows(q_out, "q_out", T)[1], _rows(k, "k", T)[1], _rows(v, "v", T)[1]
    rot = _positions(positions, freqs, T, D)
    rc = getattr(lib, name)(q_out.data_ptr(), q.data_ptr(), k.data_ptr(), v.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(),
                            slot_mapping.data_ptr(), positions.data_ptr(), freqs.data_ptr(), T, Hq, Hkv, D, rot, bool(interleaved),
                            magnitude, bs, qos, qs, ks, vs, *scales, _pkg._dtype_code(q), _pkg._stream(stream))
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
    """optgqa_common_prefix_workspace_bytes."""
    return int(_pkg.load_library().optgqa_common_prefix_workspace_bytes(num_tokens, num_seqs, num_heads, num_kv_heads, head_dim, block_size,
                                                                        num_prefix_blocks, max_context_len, max_q_len))


def _common(name, out, q, k_cache, v_cache, prefix_table, block_tables, context_lens, cu_q_lens, alibi_slopes, scale, max_context_len,
            max_q_len, workspace, stream, kv8, scales) -> None:
    lib = _pkg.load_library()
    _pkg._attn_typed(q, out, k_cache, v_cache, block_tables, context_lens, alibi_slopes, kv8=kv8, cu_q_lens=cu_q_lens)
    _pkg._typed(q, i32=(("prefix_table", prefix_table),))
    T, Hq, D = q.shape
    NB, Hkv, bs, Dk = k_cache.shape
    B = context_lens.shape[0]
    if (Dk != D or out.shape != q.shape or v_cache.shape != k_cache.shape or prefix_table.dim() != 1 or block_tables.dim() != 2
            or block_tables.shape[0] != B or (T != B if cu_q_lens is None else cu_q_lens.shape != (B + 1,))
            or (alibi_slopes is not None and alibi_slopes.shape != (Hq,))):
        raise ValueError("optgqa: shape mismatch between q, out, the tables, lengths, slopes and the caches")
    for t, n in ((out, "out"), (q, "q"), (k_cache, "k_cache"), (v_cache, "v_cache"), (prefix_table, "prefix_table"),
                 (block_tables, "block_tables"), (context_lens, "context_lens"), (cu_q_lens, "cu_q_lens"), (alibi_slopes, "alibi_slopes")):
        if t is not None:
            _pkg._dense(t, n)
    ws_bytes = _pkg._workspace(workspace, q)
    rc = getattr(lib, name)(out.data_ptr(), q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(), prefix_table.data_ptr(),
                            block_tables.data_ptr(), context_lens.data_ptr(), _pkg._ptr(cu_q_lens), _pkg._ptr(alibi_slopes), scale, *scales,
                            T, B, Hq, Hkv, D, bs, prefix_table.shape[0], block_tables.shape[1], max_context_len, max_q_len,
                            _pkg._ptr(workspace), ws_bytes, _pkg._dtype_code(q), _pkg._stream(stream))
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
    if target_probs.dtype not in _PROBABILITIES:
        raise TypeError(f"optgqa: probabilities must be float32, float16 or bfloat16, got {target_probs.dtype}")
    if draft_probs is not None and draft_probs.dtype != target_probs.dtype:
        raise TypeError(f"optgqa: draft_probs must be {target_probs.dtype}, got {draft_probs.dtype}")
    index = target_probs.get_device()
    for t, name, want in ((tokens, "tokens", torch.int64), (num_accepted, "num_accepted", torch.int32), (draft_tokens, "draft_tokens", torch.int64),
                          (cu_draft_lens, "cu_draft_lens", torch.int32), (accept_uniforms, "accept_uniforms", torch.float32),
                          (sample_uniforms, "sample_uniforms", torch.float32)):
        if t.dtype != want:
            raise TypeError(f"optgqa: {name} must be {want}, got {t.dtype}")
        if not t.is_cuda or t.get_device() != index or not t.is_contiguous():
            raise ValueError(f"optgqa: {name} must be a dense tensor on the probabilities' GPU")
    if draft_probs is not None and draft_probs.get_device() != index:
        raise ValueError("optgqa: draft_probs must be on the same GPU as target_probs")
    B, T = num_accepted.shape[0], draft_tokens.shape[0]
    if target_probs.dim() != 2 or tokens.dim() != 2:
        raise ValueError("optgqa: tokens and target_probs must have two dimensions")
    V = target_probs.shape[1]
    if (tokens.shape[0] != B or tokens.shape[1] < 1 or target_probs.shape[0] != T + B or cu_draft_lens.shape != (B + 1,)
            or accept_uniforms.shape != (T,) or sample_uniforms.shape != (B,) or (draft_probs is not None and draft_probs.shape != (T, V))):
        raise ValueError("optgqa: shape mismatch between the tokens, probabilities, drafts and random numbers")
    for t, name in ((target_probs, "target_probs"), (draft_probs, "draft_probs")):
        if t is not None and t.shape[0] and t.stride(1) != 1 and V > 1:
            raise ValueError(f"optgqa: {name} must have dense rows")
    ws_bytes = _pkg._workspace(workspace, target_probs)
    rc = lib.optgqa_verify_drafts(tokens.data_ptr(), num_accepted.data_ptr(), target_probs.data_ptr(), _pkg._ptr(draft_probs),
                                  draft_tokens.data_ptr(), cu_draft_lens.data_ptr(), accept_uniforms.data_ptr(), sample_uniforms.data_ptr(),
                                  B, V, tokens.shape[1] - 1, _row_stride(target_probs), 0 if draft_probs is None else _row_stride(draft_probs),
                                  _pkg._ptr(workspace), ws_bytes, _PROBABILITIES[target_probs.dtype], _pkg._stream(stream))
    _pkg._check(rc, "optgqa_verify_drafts")


def _row_stride(t: torch.Tensor) -> int:
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]
