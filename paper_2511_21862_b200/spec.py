"""Binding of the speculative-decoding ABI (`include/ooco_spec.h`): argument marshalling only.

As in `binding`, every function takes torch tensors whose memory the caller owns and raises `OocoError` on a non-zero
status; a tensor of the wrong type, shape, layout or device raises `ValueError`.  All tensors of a call live on one
device; the call runs there, on `stream` or that device's current stream.  The checks are in the compiled module
`_spec_calls` (csrc/py_spec.cpp), which calls the entry points of the library that `binding` has loaded.
"""
from __future__ import annotations

import ctypes
from dataclasses import dataclass, field

import torch

from . import binding
from .binding import OocoError, Shape, ooco_shape_t

TREE_MAX_NODES = 256
MAX_VOCAB = 1 << 20
STATUS_BAD_BLOCK = 4
STATUS_REFUSED = 128
ROPE_SCALINGS = {"plain": 0, "linear": 1, "stretch": 2, "bands": 3, "ramp": 4}


class ooco_rope_scaling_t(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("original_len", ctypes.c_int32), ("factor", ctypes.c_double),
                ("low", ctypes.c_double), ("high", ctypes.c_double)]


class ooco_rope_t(ctypes.Structure):
    _fields_ = [("rot_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32), ("magnitude", ctypes.c_float),
                ("reserved", ctypes.c_int32), ("inv_freq", ctypes.c_void_p)]


class ooco_verify_t(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("batch", "max_nodes", "vocab", "reserved")] + \
               [(n, ctypes.c_int64) for n in ("target_seq_stride", "target_node_stride", "draft_seq_stride",
                                              "draft_node_stride")]


_L = None        # the library whose entry points `_at` holds
_at: dict = {}   # addresses of entry points
_calls = None    # the compiled module


def _load():
    global _L, _calls
    L = binding.lib()
    if L is _L:
        return L
    if _calls is None:
        from . import build
        try:
            from . import _spec_calls
        except ImportError as e:
            raise ImportError("_spec_calls.so is missing or unusable: run `python -m paper_2511_21862_b200.build`") from e
        if _spec_calls.built_for != build._built_for():
            raise ImportError(f"_spec_calls.so was built for {_spec_calls.built_for}, this is {build._built_for()}: run "
                              "`python -m paper_2511_21862_b200.build`")
        _calls = _spec_calls
    sp, vp, i32, i64, f32, sz = (ctypes.POINTER(ooco_shape_t), ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64,
                                 ctypes.c_float, ctypes.c_size_t)
    rp, qp = ctypes.POINTER(ooco_rope_t), ctypes.POINTER(ooco_verify_t)
    rope, tree = [sp, rp, i32, vp, i64, vp, i64, vp, i64, vp, vp, vp, i64, vp, vp], [sp, i32] + [vp] * 7 + [f32]
    for name, args in (
            ("ooco_plan_slots", [sp] + [vp] * 5 + [i32, vp, vp, vp, i32, i32] + [vp] * 7 + [sz, vp, vp]),
            ("ooco_rope_frequencies", [i32, ctypes.c_double, ctypes.POINTER(ooco_rope_scaling_t), vp, vp]),
            ("ooco_rope_kv_append", rope + [vp]), ("ooco_rope_kv_append_fp8", rope + [f32, f32, vp]),
            ("ooco_tree_attention", tree + [vp, vp, sz, vp]), ("ooco_tree_attention_fp8", tree + [f32, f32, vp, vp, sz, vp]),
            ("ooco_verify_drafts", [qp] + [vp] * 10), ("ooco_kv_keep_path", [sp, i32] + [vp] * 8),
            ("ooco_kv_keep_path_fp8", [sp, i32] + [vp] * 8)):
        f = getattr(L, name)
        f.restype, f.argtypes = ctypes.c_int, args
        _at[name] = ctypes.cast(f, vp).value
    for name, args in (("ooco_plan_slots_workspace_bytes", [sp]), ("ooco_tree_workspace_bytes", [sp, i32])):
        f = getattr(L, name)
        f.restype, f.argtypes = sz, args
    _L = L
    return L


def _lib():
    return _L if _L is not None and _L is binding._lib else _load()


def _shape(shape: Shape):
    """The C struct of an (immutable) Shape, made once per object."""
    c = shape.__dict__.get("_c_struct")
    if c is None:
        c = shape.__dict__.setdefault("_c_struct", shape.c())   # (the first of several threads' stays)
    return c


def _address(shape: Shape) -> int:
    """Where this object's own struct lies: asked each time, since a copied or unpickled Shape has another."""
    return ctypes.addressof(_shape(shape))


def plan_slots_workspace_bytes(shape: Shape) -> int:
    n = _lib().ooco_plan_slots_workspace_bytes(ctypes.byref(_shape(shape)))
    if n == 0:
        raise OocoError(-3, "ooco_plan_slots_workspace_bytes")
    return int(n)


def plan_slots(shape: Shape, context_lens, new_lens, block_table, blocks_held, free_ids, free_head, slot_map, positions,
               first_token, granted_lens, total_lens, workspace, *, row_len=0, parents=None, blocks_held_out=None,
               free_head_out=None, status=None, stream=None):
    """Blocks, cache slots and positions of the tokens that every sequence adds (`row_len` = 0: packed rows, else padded
    rows of that length).  All tensors int32; `blocks_held` and `free_head` are updated in place unless outputs are given;
    no other output may share memory with an input or another output."""
    _lib()
    rc = _calls.plan_slots(_at["ooco_plan_slots"], _address(shape), context_lens, new_lens, block_table, blocks_held, free_ids,
                           free_head, blocks_held_out, free_head_out, row_len, parents, slot_map, positions, first_token,
                           granted_lens, total_lens, workspace, status, stream)
    if rc:
        raise OocoError(rc, "ooco_plan_slots")


def rope_frequencies(rot_dim: int, base: float = 10000.0, scaling: str = "plain", *, factor: float = 1.0,
                     original_len: int = 0, low: float = 0.0, high: float = 0.0):
    """(fp32 CPU tensor [rot_dim / 2], magnitude): frequencies scaled for long contexts (see OOCO_ROPE_*)."""
    inv = torch.empty(rot_dim // 2, dtype=torch.float32)
    mag = ctypes.c_float(0.0)
    sc = ooco_rope_scaling_t(ROPE_SCALINGS[scaling], int(original_len), float(factor), float(low), float(high))
    rc = _lib().ooco_rope_frequencies(int(rot_dim), float(base), ctypes.byref(sc), inv.data_ptr(), ctypes.addressof(mag))
    if rc:
        raise OocoError(rc, "ooco_rope_frequencies")
    return inv, float(mag.value)


@dataclass(frozen=True)
class Rope:
    """Rotary positions: the leading `rot_dim` dims of every head turn, `inv_freq` is fp32 [rot_dim / 2] on the device."""
    rot_dim: int
    interleaved: bool
    inv_freq: torch.Tensor
    magnitude: float = 1.0
    _c: object = field(default=None, init=False, repr=False, compare=False)

    def __post_init__(self):
        f = self.inv_freq
        if not f.is_cuda or f.dtype != torch.float32 or not f.is_contiguous() or f.numel() != self.rot_dim // 2:
            raise ValueError(f"inv_freq: expected a contiguous float32 CUDA tensor of {self.rot_dim // 2} elements, got "
                             f"{f.dtype} {tuple(f.shape)} on {f.device}")
        # (the address of inv_freq is filled in by each call, from the tensor that it has then)
        object.__setattr__(self, "_c", ooco_rope_t(self.rot_dim, int(self.interleaved), self.magnitude, 0, None))

    def __reduce__(self):  # copies and pickles are made anew, with a struct of their own
        return type(self), (self.rot_dim, self.interleaved, self.inv_freq, self.magnitude)

    @property
    def _address(self) -> int:
        return ctypes.addressof(self._c)


def rope_kv_append(shape: Shape, rope: Rope, q, k, v, positions, slot_map, q_out, k_cache, v_cache, stream=None):
    """q_out = rotated q (q itself, or memory that neither q nor k nor v has); rotated k and v go to the bf16 caches' slots.
    q, k, v: bf16 [T, heads, head_dim], views with dense rows allowed; positions, slot_map: int32 [T]."""
    _lib()
    rc = _calls.rope_kv_append(_at["ooco_rope_kv_append"], False, _address(shape), rope._address, rope.inv_freq, q, k, v,
                               positions, slot_map, q_out, k_cache, v_cache, 1.0, 1.0, stream)
    if rc:
        raise OocoError(rc, "ooco_rope_kv_append")


def rope_kv_append_fp8(shape: Shape, rope: Rope, q, k, v, positions, slot_map, q_out, k_cache, v_cache, k_scale, v_scale,
                       stream=None):
    """The same into uint8 (E4M3) caches."""
    _lib()
    rc = _calls.rope_kv_append(_at["ooco_rope_kv_append_fp8"], True, _address(shape), rope._address, rope.inv_freq, q, k, v,
                               positions, slot_map, q_out, k_cache, v_cache, k_scale, v_scale, stream)
    if rc:
        raise OocoError(rc, "ooco_rope_kv_append_fp8")


def tree_workspace_bytes(shape: Shape, max_nodes: int) -> int:
    n = _lib().ooco_tree_workspace_bytes(ctypes.byref(_shape(shape)), int(max_nodes))
    if n == 0:
        raise OocoError(-3, "ooco_tree_workspace_bytes")
    return int(n)


def _tree(name, fp8, shape, q, k_cache, v_cache, block_table, context_lens, parents, tree_sizes, scale, k_scale, v_scale, out,
          workspace, stream):
    rc = _calls.tree_attention(_at[name], fp8, _lib().ooco_get_tuning(13) != 0, _address(shape), q, k_cache, v_cache,
                               block_table, context_lens, parents, tree_sizes, scale, k_scale, v_scale, out, workspace, stream)
    if rc:
        raise OocoError(rc, name)


def tree_attention(shape: Shape, q, k_cache, v_cache, block_table, context_lens, parents, scale, out, workspace,
                   tree_sizes=None, stream=None):
    """Attention of draft trees: q, out bf16 [B, N, Hq, D]; the last tree_sizes[b] (default N) tokens of a context are
    its tree's nodes, parents int32 [B, N]; node i sees the context before the tree, its ancestors and itself."""
    _lib()
    _tree("ooco_tree_attention", False, shape, q, k_cache, v_cache, block_table, context_lens, parents, tree_sizes, scale, 1.0,
          1.0, out, workspace, stream)


def tree_attention_fp8(shape: Shape, q, k_cache, v_cache, block_table, context_lens, parents, scale, k_scale, v_scale, out,
                       workspace, tree_sizes=None, stream=None):
    """The same over uint8 (E4M3) caches."""
    _lib()
    _tree("ooco_tree_attention_fp8", True, shape, q, k_cache, v_cache, block_table, context_lens, parents, tree_sizes, scale,
          k_scale, v_scale, out, workspace, stream)


def verify_drafts(target_probs, draft_probs, tokens, parents, uniforms, path, out_tokens, num_accepted, tree_sizes=None,
                  stream=None):
    """Walks each sequence's draft tree against the target's probabilities.  target_probs, draft_probs: fp32 [B, N, V]
    (draft_probs None: drafts chosen, not drawn); tokens, parents (None: a chain), path, out_tokens: int32 [B, N];
    uniforms fp32 [B, N]; num_accepted, tree_sizes (None: N): int32 [B]."""
    _lib()
    rc = _calls.verify_drafts(_at["ooco_verify_drafts"], target_probs, draft_probs, tokens, parents, uniforms, path, out_tokens,
                              num_accepted, tree_sizes, stream)
    if rc:
        raise OocoError(rc, "ooco_verify_drafts")


def kv_keep_path(shape: Shape, k_cache, v_cache, block_table, base_lens, path, num_accepted, context_lens_out=None,
                 stream=None):
    """Moves the accepted branch's cache rows (tokens base + path[b, j]) to tokens base + j; context_lens_out: the new
    context lengths."""
    _lib()
    rc = _calls.kv_keep_path(_at["ooco_kv_keep_path"], False, _address(shape), k_cache, v_cache, block_table, base_lens, path,
                             num_accepted, context_lens_out, stream)
    if rc:
        raise OocoError(rc, "ooco_kv_keep_path")


def kv_keep_path_fp8(shape: Shape, k_cache, v_cache, block_table, base_lens, path, num_accepted, context_lens_out=None,
                     stream=None):
    """The same for uint8 (E4M3) caches."""
    _lib()
    rc = _calls.kv_keep_path(_at["ooco_kv_keep_path_fp8"], True, _address(shape), k_cache, v_cache, block_table, base_lens, path,
                             num_accepted, context_lens_out, stream)
    if rc:
        raise OocoError(rc, "ooco_kv_keep_path_fp8")
