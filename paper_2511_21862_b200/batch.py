"""Binding of the continuous-batching ABI (`include/ooco_batch.h`): argument marshalling only, as in `spec`.

Between steps `fork_pages` and `release_pages` share and give back cache pages; a step runs `spec.plan_slots` (packed rows),
then per layer `norm_rope_kv_append` (or `spec.rope_kv_append`) and `chunk_attention`, and at its end `shape_logits`, whose
probabilities `spec.verify_drafts` or a sampler takes.  Every function takes torch tensors whose memory the caller owns and
raises `OocoError` on a non-zero status; a tensor of the wrong type, shape, layout or device raises `ValueError`.  All tensors
of a call live on one device; the call runs there, on `stream` or that device's current stream.
"""
from __future__ import annotations

import ctypes
from dataclasses import dataclass, field

import torch

from . import binding, spec
from .binding import OocoError, Shape, ooco_shape_t
from .spec import Rope, ooco_rope_t

MAX_PAGE_ROWS = 1 << 18
MAX_SHAPED_VOCAB = 409600
MAX_BIAS = 1024


class ooco_head_norm_t(ctypes.Structure):
    _fields_ = [("eps", ctypes.c_float), ("weight_offset", ctypes.c_float), ("q_weight", ctypes.c_void_p),
                ("k_weight", ctypes.c_void_p)]


class ooco_logits_t(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("batch", "max_nodes", "vocab", "logits_fp32", "history_width", "max_bias")] + \
               [(n, ctypes.c_int64) for n in ("logits_seq_stride", "logits_node_stride", "out_seq_stride", "out_node_stride",
                                              "probs_seq_stride", "probs_node_stride", "mask_seq_stride", "mask_node_stride")]


_L = None        # the library whose entry points `_at` holds
_at: dict = {}   # addresses of entry points
_calls = None    # the compiled module


def _load():
    global _L, _calls
    L = spec._lib()
    _calls = spec._calls
    sp, vp, i32, i64, f32, sz = (ctypes.POINTER(ooco_shape_t), ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64,
                                 ctypes.c_float, ctypes.c_size_t)
    norm = [sp, ctypes.POINTER(ooco_rope_t), ctypes.POINTER(ooco_head_norm_t), i32, vp, i64, vp, i64, vp, i64, vp, vp, vp, i64,
            vp, vp]
    chunk = [sp, i32, i32, vp, i64] + [vp] * 6 + [f32]
    for name, args in (
            ("ooco_fork_pages", [sp, i32] + [vp] * 7 + [i32] + [vp] * 10 + [sz, vp, vp]),
            ("ooco_release_pages", [sp, i32] + [vp] * 6 + [i32] + [vp] * 7 + [sz, vp, vp]),
            ("ooco_norm_rope_kv_append", norm + [vp]), ("ooco_norm_rope_kv_append_fp8", norm + [f32, f32, vp]),
            ("ooco_shape_logits", [ctypes.POINTER(ooco_logits_t)] + [vp] * 17),
            ("ooco_chunk_attention", chunk + [vp, i64, vp, sz, vp]),
            ("ooco_chunk_attention_fp8", chunk + [f32, f32, vp, i64, vp, sz, vp])):
        f = getattr(L, name)
        f.restype, f.argtypes = ctypes.c_int, args
        _at[name] = ctypes.cast(f, vp).value
    for name, args in (("ooco_pages_workspace_bytes", [sp, i32]), ("ooco_chunk_workspace_bytes", [sp, i32, i32])):
        f = getattr(L, name)
        f.restype, f.argtypes = sz, args
    _L = L
    return L


def _lib():
    return _L if _L is not None and _L is binding._lib else _load()


def _done(rc: int, name: str):
    if rc:
        raise OocoError(rc, name)


def pages_workspace_bytes(shape: Shape, num_rows: int) -> int:
    n = _lib().ooco_pages_workspace_bytes(ctypes.byref(spec._shape(shape)), int(num_rows))
    if n == 0:
        raise OocoError(-3, "ooco_pages_workspace_bytes")
    return int(n)


def fork_pages(shape: Shape, parents, children, context_lens, block_table, blocks_held, free_ids, free_head, shares, copy_src,
               copy_dst, granted, workspace, *, shared_lens=None, context_lens_out=None, blocks_held_out=None,
               free_head_out=None, shares_out=None, status=None, stream=None):
    """Row children[c] gets the first tokens of row parents[c] (all, or shared_lens[c]): full pages are shared, a partly filled
    last one is a page of its own, to be copied by `binding.kv_copy_blocks(shape, ..., copy_src, copy_dst)`.  All tensors int32;
    lengths, pages held, the list's head and the holder counts are updated in place unless outputs are given."""
    _lib()
    _done(_calls.fork_pages(_at["ooco_fork_pages"], spec._address(shape), parents, children, shared_lens, context_lens,
                            block_table, blocks_held, free_ids, free_head, shares, context_lens_out, blocks_held_out,
                            free_head_out, shares_out, copy_src, copy_dst, granted, workspace, status, stream),
          "ooco_fork_pages")


def release_pages(shape: Shape, rows, context_lens, block_table, blocks_held, free_ids, free_head, shares, workspace, *,
                  keep_lens=None, context_lens_out=None, blocks_held_out=None, free_head_out=None, shares_out=None, status=None,
                  stream=None):
    """Row rows[c] keeps its first keep_lens[c] tokens (None: nothing); pages that no other row holds go back to the free list,
    in front of its head.  All tensors int32; updated in place unless outputs are given."""
    _lib()
    _done(_calls.release_pages(_at["ooco_release_pages"], spec._address(shape), rows, keep_lens, context_lens, block_table,
                               blocks_held, free_ids, free_head, shares, context_lens_out, blocks_held_out, free_head_out,
                               shares_out, workspace, status, stream), "ooco_release_pages")


@dataclass(frozen=True)
class HeadNorm:
    """Norms of the heads of q and k: bf16 weights [head_dim] on the device, or None; `weight_offset` is added to them."""
    eps: float
    q_weight: torch.Tensor | None = None
    k_weight: torch.Tensor | None = None
    weight_offset: float = 0.0
    _c: object = field(default=None, init=False, repr=False, compare=False)

    def __post_init__(self):
        for name in ("q_weight", "k_weight"):
            w = getattr(self, name)
            if w is not None and (not w.is_cuda or w.dtype != torch.bfloat16 or not w.is_contiguous() or w.dim() != 1):
                raise ValueError(f"{name}: expected a contiguous bfloat16 CUDA vector, got {w.dtype} {tuple(w.shape)} on {w.device}")
        # (the weights' addresses are filled in by each call, from the tensors that it has then)
        object.__setattr__(self, "_c", ooco_head_norm_t(self.eps, self.weight_offset, None, None))

    def __reduce__(self):  # copies and pickles are made anew, with a struct of their own
        return type(self), (self.eps, self.q_weight, self.k_weight, self.weight_offset)

    @property
    def _address(self) -> int:
        return ctypes.addressof(self._c)


def _norm_rope(name, fp8, shape, rope, norm, q, k, v, positions, slot_map, q_out, k_cache, v_cache, k_scale, v_scale, stream):
    _lib()
    _done(_calls.norm_rope_kv_append(_at[name], fp8, spec._address(shape), rope._address, rope.inv_freq, norm._address,
                                     norm.q_weight, norm.k_weight, q, k, v, positions, slot_map, q_out, k_cache, v_cache,
                                     k_scale, v_scale, stream), name)


def norm_rope_kv_append(shape: Shape, rope: Rope, norm: HeadNorm, q, k, v, positions, slot_map, q_out, k_cache, v_cache,
                        stream=None):
    """`spec.rope_kv_append` with a norm of every head of q and k before the rotation."""
    _norm_rope("ooco_norm_rope_kv_append", False, shape, rope, norm, q, k, v, positions, slot_map, q_out, k_cache, v_cache, 1.0,
               1.0, stream)


def norm_rope_kv_append_fp8(shape: Shape, rope: Rope, norm: HeadNorm, q, k, v, positions, slot_map, q_out, k_cache, v_cache,
                            k_scale, v_scale, stream=None):
    """The same into uint8 (E4M3) caches."""
    _norm_rope("ooco_norm_rope_kv_append_fp8", True, shape, rope, norm, q, k, v, positions, slot_map, q_out, k_cache, v_cache,
               k_scale, v_scale, stream)


def chunk_workspace_bytes(shape: Shape, num_rows: int, max_chunk: int) -> int:
    n = _lib().ooco_chunk_workspace_bytes(ctypes.byref(spec._shape(shape)), int(num_rows), int(max_chunk))
    if n == 0:
        raise OocoError(-3, "ooco_chunk_workspace_bytes")
    return int(n)


def _chunk(name, fp8, shape, q, k_cache, v_cache, block_table, context_lens, first_row, max_chunk, scale, k_scale, v_scale, out,
           workspace, chunk_lens, stream):
    _lib()
    _done(_calls.chunk_attention(_at[name], fp8, spec._address(shape), q, k_cache, v_cache, block_table, context_lens, first_row,
                                 max_chunk, scale, k_scale, v_scale, out, workspace, chunk_lens, stream), name)


def chunk_attention(shape: Shape, q, k_cache, v_cache, block_table, context_lens, first_row, max_chunk, scale, out, workspace,
                    chunk_lens=None, stream=None):
    """Causal attention of all sequences' new tokens, packed: q, out bf16 [rows, Hq, D] (views with dense rows allowed), those of
    sequence b from row first_row[b] on, the last first_row[b + 1] - first_row[b] (or chunk_lens[b], if smaller) tokens of its
    context_lens[b]; none brings more than max_chunk."""
    _chunk("ooco_chunk_attention", False, shape, q, k_cache, v_cache, block_table, context_lens, first_row, max_chunk, scale, 1.0,
           1.0, out, workspace, chunk_lens, stream)


def chunk_attention_fp8(shape: Shape, q, k_cache, v_cache, block_table, context_lens, first_row, max_chunk, scale, k_scale,
                        v_scale, out, workspace, chunk_lens=None, stream=None):
    """The same over uint8 (E4M3) caches."""
    _chunk("ooco_chunk_attention_fp8", True, shape, q, k_cache, v_cache, block_table, context_lens, first_row, max_chunk, scale,
           k_scale, v_scale, out, workspace, chunk_lens, stream)


def shape_logits(logits, *, out=None, probs=None, temperature=None, repetition=None, frequency=None, presence=None, history=None,
                 history_lens=None, prompt_lens=None, tokens=None, parents=None, tree_sizes=None, bias_tokens=None,
                 bias_values=None, mask=None, stream=None):
    """Penalties for repeated tokens, biases and masks on logits (bf16 or fp32, [B, V] or [B, N, V] for the nodes of draft
    trees): the shaped logits to `out`, their softmax at `temperature` to `probs` (fp32, logits' shape; fp32 logits may be one of
    them).  temperature, repetition, frequency, presence: fp32 [B]; history: int32 [B, L] with history_lens and prompt_lens [B];
    tokens, parents: int32 [B, N]; bias_tokens int32 and bias_values fp32 [B, M]; mask: int32 words [B, (N,) ceil(V / 32)],
    expanded dimensions allowed."""
    _lib()
    _done(_calls.shape_logits(_at["ooco_shape_logits"], logits, out, probs, temperature, repetition, frequency, presence, history,
                              history_lens, prompt_lens, tokens, parents, tree_sizes, bias_tokens, bias_values, mask, stream),
          "ooco_shape_logits")
