"""ctypes binding of the speculative-decoding ABI (`include/ooco_spec.h`): argument marshalling only.

As in `binding`, every function takes torch tensors whose memory the caller owns and raises `OocoError` on a non-zero
status.  All tensors of a call live on one device; the call runs there, on `stream` or that device's current stream.
"""
from __future__ import annotations

import ctypes
from dataclasses import dataclass, field

import torch

from .binding import OocoError, Shape, get_tuning, lib, ooco_shape_t

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


_L = None


def _lib():
    global _L
    L = lib()
    if L is not _L:
        sp, vp, i32, i64, f32, sz = (ctypes.POINTER(ooco_shape_t), ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64,
                                     ctypes.c_float, ctypes.c_size_t)
        rp, qp = ctypes.POINTER(ooco_rope_t), ctypes.POINTER(ooco_verify_t)
        L.ooco_plan_slots_workspace_bytes.restype = sz
        L.ooco_plan_slots_workspace_bytes.argtypes = [sp]
        L.ooco_plan_slots.restype = ctypes.c_int
        L.ooco_plan_slots.argtypes = [sp, vp, vp, vp, vp, vp, i32, vp, vp, vp, i32, i32, vp, vp, vp, vp, vp, vp, vp, sz, vp,
                                      vp]
        L.ooco_rope_frequencies.restype = ctypes.c_int
        L.ooco_rope_frequencies.argtypes = [i32, ctypes.c_double, ctypes.POINTER(ooco_rope_scaling_t), vp, vp]
        rope = [sp, rp, i32, vp, i64, vp, i64, vp, i64, vp, vp, vp, i64, vp, vp]
        L.ooco_rope_kv_append.restype = ctypes.c_int
        L.ooco_rope_kv_append.argtypes = rope + [vp]
        L.ooco_rope_kv_append_fp8.restype = ctypes.c_int
        L.ooco_rope_kv_append_fp8.argtypes = rope + [f32, f32, vp]
        L.ooco_tree_workspace_bytes.restype = sz
        L.ooco_tree_workspace_bytes.argtypes = [sp, i32]
        tree = [sp, i32, vp, vp, vp, vp, vp, vp, vp, f32]
        L.ooco_tree_attention.restype = ctypes.c_int
        L.ooco_tree_attention.argtypes = tree + [vp, vp, sz, vp]
        L.ooco_tree_attention_fp8.restype = ctypes.c_int
        L.ooco_tree_attention_fp8.argtypes = tree + [f32, f32, vp, vp, sz, vp]
        L.ooco_verify_drafts.restype = ctypes.c_int
        L.ooco_verify_drafts.argtypes = [qp] + [vp] * 10
        for f in (L.ooco_kv_keep_path, L.ooco_kv_keep_path_fp8):
            f.restype = ctypes.c_int
            f.argtypes = [sp, i32] + [vp] * 8
        _L = L
    return L


def _shape(shape: Shape):
    """The C struct of an (immutable) Shape, made once per object."""
    c = shape.__dict__.get("_c_ref")
    if c is None:
        c = ctypes.byref(shape.c())
        object.__setattr__(shape, "_c_ref", c)
    return c


def _call(name, dev, stream, *args):
    """Calls `name` with the stream's pointer behind `args`, on device `dev`."""
    if stream is None:
        stream = torch.cuda.current_stream(dev)
    if dev != torch.cuda.current_device():
        with torch.cuda.device(dev):
            rc = getattr(_L or _lib(), name)(*args, stream.cuda_stream)
    else:
        rc = getattr(_L or _lib(), name)(*args, stream.cuda_stream)
    if rc:
        raise OocoError(rc, name)


def _ptr(t, dev, dtype, what, shape=None):
    """Address of a contiguous tensor on device `dev`; `shape`: what its shape must be."""
    if t.get_device() != dev or t.dtype != dtype or not t.is_contiguous() or (shape is not None and t.shape != shape):
        raise ValueError(f"{what}: expected a contiguous {dtype} tensor on cuda:{dev}"
                         f"{'' if shape is None else f' of shape {tuple(shape)}'}, "
                         f"got {t.dtype} {tuple(t.shape)} on {t.device}")
    return t.data_ptr()


def _cuda(t, what):
    dev = t.get_device()
    if dev < 0:
        raise ValueError(f"{what}: expected a CUDA tensor, got one on {t.device}")
    return dev


def _room(t, count, what):
    if t.numel() < count:
        raise ValueError(f"{what}: expected at least {count} elements, got {t.numel()}")
    return t


def _pool(shape: Shape, k_cache, v_cache, dev, dtype):
    """Addresses of the two caches, which must hold the pool that `shape` describes."""
    last = ((shape.num_blocks - 1) * shape.kv_block_stride + (shape.num_kv_heads - 1) * shape.kv_head_stride +
            (shape.block_size - 1) * shape.kv_token_stride + shape.head_dim)
    return (_ptr(_room(k_cache, last, "k_cache"), dev, dtype, "k_cache"),
            _ptr(_room(v_cache, last, "v_cache"), dev, dtype, "v_cache"))


def plan_slots_workspace_bytes(shape: Shape) -> int:
    n = _lib().ooco_plan_slots_workspace_bytes(_shape(shape))
    if n == 0:
        raise OocoError(-3, "ooco_plan_slots_workspace_bytes")
    return int(n)


def plan_slots(shape: Shape, context_lens, new_lens, block_table, blocks_held, free_ids, free_head, slot_map, positions,
               first_token, granted_lens, total_lens, workspace, *, row_len=0, parents=None, blocks_held_out=None,
               free_head_out=None, status=None, stream=None):
    """Blocks, cache slots and positions of the tokens that every sequence adds (`row_len` = 0: packed rows, else padded
    rows of that length).  All tensors int32; `blocks_held` and `free_head` are updated in place unless outputs are given."""
    _lib()
    dev, i32 = _cuda(context_lens, "context_lens"), torch.int32
    B, rows = shape.batch, slot_map.numel()
    per_seq, one = torch.Size((B,)), torch.Size((1,))
    _call("ooco_plan_slots", dev, stream, _shape(shape), _ptr(context_lens, dev, i32, "context_lens", per_seq),
          _ptr(new_lens, dev, i32, "new_lens", per_seq),
          _ptr(block_table, dev, i32, "block_table", torch.Size((B, shape.max_blocks_per_seq))),
          _ptr(blocks_held, dev, i32, "blocks_held", per_seq), _ptr(free_ids, dev, i32, "free_ids"), free_ids.numel(),
          _ptr(free_head, dev, i32, "free_head", one),
          None if blocks_held_out is None else _ptr(blocks_held_out, dev, i32, "blocks_held_out", per_seq),
          None if free_head_out is None else _ptr(free_head_out, dev, i32, "free_head_out", one), row_len, rows,
          None if parents is None else _ptr(_room(parents, rows, "parents"), dev, i32, "parents"),
          _ptr(slot_map, dev, i32, "slot_map"), _ptr(_room(positions, rows, "positions"), dev, i32, "positions"),
          _ptr(first_token, dev, i32, "first_token", torch.Size((B + 1,))),
          _ptr(granted_lens, dev, i32, "granted_lens", per_seq), _ptr(total_lens, dev, i32, "total_lens", per_seq),
          _ptr(workspace, dev, torch.uint8, "workspace"), workspace.numel(),
          None if status is None else _ptr(status, dev, i32, "status", one))


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
        _ptr(f, _cuda(f, "inv_freq"), torch.float32, "inv_freq", torch.Size((self.rot_dim // 2,)))
        object.__setattr__(self, "_c", ooco_rope_t(self.rot_dim, int(self.interleaved), self.magnitude, 0, f.data_ptr()))


def _rows(t, heads, dim, tokens, dev, what):
    """(address, row stride) of bf16 rows [tokens, heads, dim], dense inside a row."""
    if (t.dim() != 3 or t.shape != (tokens, heads, dim) or t.dtype != torch.bfloat16 or t.get_device() != dev or
            t.stride(2) != 1 or t.stride(1) != dim):
        raise ValueError(f"{what}: expected bfloat16 [{tokens}, {heads}, {dim}] with dense rows on cuda:{dev}, got "
                         f"{t.dtype} {tuple(t.shape)} with strides {t.stride()} on {t.device}")
    return t.data_ptr(), t.stride(0) if tokens > 1 else max(t.stride(0), heads * dim)


def _rope(name, dtype, scales, shape, rope, q, k, v, positions, slot_map, q_out, k_cache, v_cache, stream):
    _lib()
    dev, T, D = _cuda(q, "q"), q.shape[0], shape.head_dim
    rows = torch.Size((T,))
    if rope.inv_freq.get_device() != dev:
        raise ValueError(f"inv_freq: expected a tensor on cuda:{dev}")
    _call(name, dev, stream, _shape(shape), ctypes.byref(rope._c), T, *_rows(q, shape.num_q_heads, D, T, dev, "q"),
          *_rows(k, shape.num_kv_heads, D, T, dev, "k"), *_rows(v, shape.num_kv_heads, D, T, dev, "v"),
          _ptr(positions, dev, torch.int32, "positions", rows), _ptr(slot_map, dev, torch.int32, "slot_map", rows),
          *_rows(q_out, shape.num_q_heads, D, T, dev, "q_out"), *_pool(shape, k_cache, v_cache, dev, dtype), *scales)


def rope_kv_append(shape: Shape, rope: Rope, q, k, v, positions, slot_map, q_out, k_cache, v_cache, stream=None):
    """q_out = rotated q (may be q); rotated k and v go to the bf16 caches' slots.  q, k, v: bf16 [T, heads, head_dim],
    views with dense rows allowed; positions, slot_map: int32 [T]."""
    _rope("ooco_rope_kv_append", torch.bfloat16, (), shape, rope, q, k, v, positions, slot_map, q_out, k_cache, v_cache,
          stream)


def rope_kv_append_fp8(shape: Shape, rope: Rope, q, k, v, positions, slot_map, q_out, k_cache, v_cache, k_scale, v_scale,
                       stream=None):
    """The same into uint8 (E4M3) caches."""
    _rope("ooco_rope_kv_append_fp8", torch.uint8, (float(k_scale), float(v_scale)), shape, rope, q, k, v, positions,
          slot_map, q_out, k_cache, v_cache, stream)


def tree_workspace_bytes(shape: Shape, max_nodes: int) -> int:
    n = _lib().ooco_tree_workspace_bytes(_shape(shape), int(max_nodes))
    if n == 0:
        raise OocoError(-3, "ooco_tree_workspace_bytes")
    return int(n)


def _tree(name, dtype, scales, shape, q, k_cache, v_cache, block_table, context_lens, parents, scale, out, workspace,
          tree_sizes, stream):
    _lib()
    dev, B = _cuda(q, "q"), shape.batch
    if q.dim() != 4:
        raise ValueError(f"q: expected [batch, max_nodes, q heads, head_dim], got {tuple(q.shape)}")
    N = q.shape[1]
    rows = torch.Size((B, N, shape.num_q_heads, shape.head_dim))
    out_type = torch.float32 if get_tuning("out_f32") else torch.bfloat16
    _call(name, dev, stream, _shape(shape), N, _ptr(q, dev, torch.bfloat16, "q", rows),
          *_pool(shape, k_cache, v_cache, dev, dtype),
          _ptr(block_table, dev, torch.int32, "block_table", torch.Size((B, shape.max_blocks_per_seq))),
          _ptr(context_lens, dev, torch.int32, "context_lens", torch.Size((B,))),
          _ptr(parents, dev, torch.int32, "parents", torch.Size((B, N))),
          None if tree_sizes is None else _ptr(tree_sizes, dev, torch.int32, "tree_sizes", torch.Size((B,))),
          scale, *scales, _ptr(out, dev, out_type, "out", rows), _ptr(workspace, dev, torch.uint8, "workspace"),
          workspace.numel())


def tree_attention(shape: Shape, q, k_cache, v_cache, block_table, context_lens, parents, scale, out, workspace,
                   tree_sizes=None, stream=None):
    """Attention of draft trees: q, out bf16 [B, N, Hq, D]; the last tree_sizes[b] (default N) tokens of a context are
    its tree's nodes, parents int32 [B, N]; node i sees the context before the tree, its ancestors and itself."""
    _tree("ooco_tree_attention", torch.bfloat16, (), shape, q, k_cache, v_cache, block_table, context_lens, parents, scale,
          out, workspace, tree_sizes, stream)


def tree_attention_fp8(shape: Shape, q, k_cache, v_cache, block_table, context_lens, parents, scale, k_scale, v_scale, out,
                       workspace, tree_sizes=None, stream=None):
    """The same over uint8 (E4M3) caches."""
    _tree("ooco_tree_attention_fp8", torch.uint8, (float(k_scale), float(v_scale)), shape, q, k_cache, v_cache, block_table,
          context_lens, parents, scale, out, workspace, tree_sizes, stream)


def _probs(t, B, N, V, dev, what):
    """(address, sequence stride, node stride) of fp32 rows [B, N, V]."""
    if t.shape != (B, N, V) or t.dtype != torch.float32 or t.get_device() != dev or (V > 1 and t.stride(2) != 1):
        raise ValueError(f"{what}: expected float32 [{B}, {N}, {V}] with dense rows on cuda:{dev}, got {t.dtype} "
                         f"{tuple(t.shape)} with strides {t.stride()} on {t.device}")
    return t.data_ptr(), t.stride(0), t.stride(1)


def verify_drafts(target_probs, draft_probs, tokens, parents, uniforms, path, out_tokens, num_accepted, tree_sizes=None,
                  stream=None):
    """Walks each sequence's draft tree against the target's probabilities.  target_probs, draft_probs: fp32 [B, N, V]
    (draft_probs None: drafts chosen, not drawn); tokens, parents (None: a chain), path, out_tokens: int32 [B, N];
    uniforms fp32 [B, N]; num_accepted, tree_sizes (None: N): int32 [B]."""
    _lib()
    dev = _cuda(target_probs, "target_probs")
    if target_probs.dim() != 3:
        raise ValueError(f"target_probs: expected [batch, nodes, vocabulary], got {tuple(target_probs.shape)}")
    B, N, V = target_probs.shape
    t_ptr, t_seq, t_node = _probs(target_probs, B, N, V, dev, "target_probs")
    d_ptr, d_seq, d_node = (None, 0, 0) if draft_probs is None else _probs(draft_probs, B, N, V, dev, "draft_probs")
    c = ooco_verify_t(B, N, V, 0, t_seq, t_node, d_seq, d_node)
    nodes, i32 = torch.Size((B, N)), torch.int32
    _call("ooco_verify_drafts", dev, stream, ctypes.byref(c), t_ptr, d_ptr, _ptr(tokens, dev, i32, "tokens", nodes),
          None if parents is None else _ptr(parents, dev, i32, "parents", nodes),
          None if tree_sizes is None else _ptr(tree_sizes, dev, i32, "tree_sizes", torch.Size((B,))),
          _ptr(uniforms, dev, torch.float32, "uniforms", nodes), _ptr(path, dev, i32, "path", nodes),
          _ptr(out_tokens, dev, i32, "out_tokens", nodes), _ptr(num_accepted, dev, i32, "num_accepted", torch.Size((B,))))


def _keep(name, dtype, shape, k_cache, v_cache, block_table, base_lens, path, num_accepted, context_lens_out, stream):
    _lib()
    dev, B, i32 = _cuda(path, "path"), shape.batch, torch.int32
    per_seq = torch.Size((B,))
    if path.dim() != 2 or path.shape[0] != B:
        raise ValueError(f"path: expected [{B}, max_nodes], got {tuple(path.shape)}")
    _call(name, dev, stream, _shape(shape), path.shape[1], *_pool(shape, k_cache, v_cache, dev, dtype),
          _ptr(block_table, dev, i32, "block_table", torch.Size((B, shape.max_blocks_per_seq))),
          _ptr(base_lens, dev, i32, "base_lens", per_seq), _ptr(path, dev, i32, "path"),
          _ptr(num_accepted, dev, i32, "num_accepted", per_seq),
          None if context_lens_out is None else _ptr(context_lens_out, dev, i32, "context_lens_out", per_seq))


def kv_keep_path(shape: Shape, k_cache, v_cache, block_table, base_lens, path, num_accepted, context_lens_out=None,
                 stream=None):
    """Moves the accepted branch's cache rows (tokens base + path[b, j]) to tokens base + j; context_lens_out: the new
    context lengths."""
    _keep("ooco_kv_keep_path", torch.bfloat16, shape, k_cache, v_cache, block_table, base_lens, path, num_accepted,
          context_lens_out, stream)


def kv_keep_path_fp8(shape: Shape, k_cache, v_cache, block_table, base_lens, path, num_accepted, context_lens_out=None,
                     stream=None):
    """The same for uint8 (E4M3) caches."""
    _keep("ooco_kv_keep_path_fp8", torch.uint8, shape, k_cache, v_cache, block_table, base_lens, path, num_accepted,
          context_lens_out, stream)
