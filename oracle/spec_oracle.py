"""Plain definitions of the speculative-decoding operators, in Python and 64-bit numpy (test infrastructure).

Written from the definitions, one sequence (one row, one node) at a time; nothing is shared with the CUDA sources.
"""
from __future__ import annotations

import math

import numpy as np


def plan_slots(ctx, new, table, held, free_ids, head, *, block_size, num_blocks, row_len, num_rows, parents=None):
    """Sequence by sequence.  Returns a dict of what the call writes (table is a changed copy)."""
    B, MB = table.shape
    ctx, new = np.maximum(ctx, 0).astype(np.int64), np.maximum(new, 0).astype(np.int64)
    held = np.clip(held, 0, MB).astype(np.int64)
    table = table.copy()
    slots, pos = np.full(num_rows, -1, np.int64), np.full(num_rows, -1, np.int64)
    first, granted, total, held_out = np.zeros(B + 1, np.int64), np.zeros(B, np.int64), ctx.copy(), held.copy()
    at, head = 0, max(0, int(head))
    start_head, promised, refused, bad = head, 0, False, False
    for b in range(B):
        row0 = b * row_len if row_len else at
        first[b] = min(row0, num_rows)
        at += int(new[b])
        room = new[b] == 0 or (new[b] <= row_len if row_len else at <= num_rows)
        fits = room and ctx[b] + new[b] <= MB * block_size and ctx[b] <= held[b] * block_size
        need = max(0, -(-int(ctx[b] + new[b]) // block_size) - int(held[b])) if fits else 0
        promised += need
        ok = fits and (need == 0 or start_head + promised <= len(free_ids))
        refused |= not ok
        if ok:
            for j in range(need):
                table[b, held[b] + j] = free_ids[start_head + promised - need + j]
            held_out[b] += need
            granted[b], total[b] = new[b], ctx[b] + new[b]
            if need:
                head = start_head + promised
        for i in range(int(new[b])):
            r = row0 + i
            if r >= num_rows or (row_len and i >= row_len):
                break
            depth = i
            if parents is not None:
                depth, j = 0, i
                while 0 <= parents[row0 + j] < j:
                    j = int(parents[row0 + j])
                    depth += 1
            pos[r] = ctx[b] + depth
            if ok:
                t = int(ctx[b]) + i
                blk = int(table[b, t // block_size])
                if 0 <= blk < num_blocks:
                    slots[r] = blk * block_size + t % block_size
                else:
                    bad = True
    first[B] = num_rows if row_len else min(at, num_rows)
    return dict(table=table, slot_map=slots, positions=pos, first_token=first, granted=granted, total=total, held=held_out,
                head=head, status=(128 if refused else 0) | (4 if bad else 0))


def rope(x, positions, inv_freq, rot_dim, interleaved, magnitude):
    """x: fp64 [T, H, D].  Pair by pair, as a rotation of a complex number."""
    y = x.astype(np.float64).copy()
    for r, p in enumerate(positions):
        for j in range(rot_dim // 2):
            a, b = (2 * j, 2 * j + 1) if interleaved else (j, j + rot_dim // 2)
            z = (y[r, :, a] + 1j * y[r, :, b]) * (magnitude * np.exp(1j * (float(p) * float(inv_freq[j]))))
            y[r, :, a], y[r, :, b] = z.real, z.imag
    return y


def sees(parents, i):
    """The nodes that node i attends to: itself and everything above it."""
    out, j = {i}, i
    while 0 <= parents[j] < j:
        j = int(parents[j])
        out.add(j)
    return out


def tree_attention(q, k, v, parents, n, scale):
    """One sequence and kv head: q [n, G, D], k and v [T, D] of the whole context (the last n tokens are the nodes), all
    fp64.  Returns (out [n, G, D], sum of |weight * value| [n, G, D], largest sum of |q_d k_d| * scale of a token seen)."""
    T = k.shape[0]
    out, mag = np.zeros(q.shape), np.zeros(q.shape)
    spread = np.zeros(q.shape[:2])
    for i in range(n):
        tok = [t for t in range(T) if t < T - n] + [T - n + j for j in sorted(sees(parents, i)) if T - n + j >= 0]
        if not tok:
            continue
        s = (q[i] @ k[tok].T) * scale
        w = np.exp(s - s.max(-1, keepdims=True))
        w /= w.sum(-1, keepdims=True)
        out[i], mag[i] = w @ v[tok], w @ np.abs(v[tok])
        spread[i] = (np.abs(q[i]) @ np.abs(k[tok]).T).max(-1) * scale
    return out, mag, spread


def verify(p, q, tokens, parents, n, uniforms):
    """One sequence: p, q (or None) fp32 [N, V].  Returns (path, out_tokens, accepted, margin); margin is how far the
    nearest comparison was from going the other way, relative to its larger side."""
    N, V = p.shape
    path, out = np.full(N, -1), np.full(N, -1)
    if n <= 0:
        return path, out, 0, math.inf
    margin = math.inf

    def less(a, b):
        nonlocal margin
        if a != b:
            margin = min(margin, abs(a - b) / max(abs(a), abs(b)))
        return a < b

    def parent(i):
        up = i - 1 if parents is None else int(parents[i])
        return up if 0 <= up < i and 0 <= tokens[i] < V else -1

    cur, count = 0, 0
    path[0] = 0
    if q is not None:
        q = np.where(q > 0, q, np.float32(0))  # (NaN and negative values count as nothing)
    while True:
        w = np.where(p[cur] > 0, p[cur], 0).astype(np.float64)  # (NaN counts as nothing)
        mass, chosen = 1.0, None
        base = w.copy()
        for c in range(cur + 1, n):
            if parent(c) != cur:
                continue
            x = int(tokens[c])
            qx = 1.0 if q is None else float(q[cur, x])
            if less(float(uniforms[c]) * mass * qx, float(w[x])):
                chosen = c
                break
            if q is None:
                mass -= w[x]
                w[x] = 0.0
            else:
                w = np.maximum(w - mass * q[cur].astype(np.float64), 0.0)
                mass = float(np.sum(w))
        if chosen is None:
            break
        cur, count = chosen, count + 1
        path[count], out[count - 1] = chosen, tokens[chosen]
    if not (w.sum() > 0 and np.isfinite(w.sum())):
        w = base
    total = float(w.sum())
    if not (total > 0 and np.isfinite(total)):
        out[count] = 0
        return path, out, count, margin
    acc = np.cumsum(w)
    t = float(uniforms[0]) * total
    at = int(np.searchsorted(acc, t, side="right"))
    out[count] = min(at, V - 1)
    for edge in (acc[at - 1] if at else -1.0, acc[min(at, V - 1)]):
        margin = min(margin, abs(edge - t) / total)
    return path, out, count, margin


def keep_path(pool, table, base, path, accepted, block_size):
    """pool: [NB, Hkv, bs, ...] (changed in place).  Returns the new context lengths."""
    NB, (B, MB), N = pool.shape[0], table.shape, path.shape[1]
    new = np.maximum(base, 0).astype(np.int64)
    for b in range(B):
        if path[b, 0] != 0:
            continue
        j, moves = 1, []
        while j <= min(max(0, accepted[b]), N - 1) and path[b, j - 1] < path[b, j] < N:
            moves.append((max(0, int(base[b])) + int(path[b, j]), max(0, int(base[b])) + j))
            j += 1
        new[b] += j
        for src, dst in moves:
            if src == dst or src >= MB * block_size:
                continue
            bs_, bd = int(table[b, src // block_size]), int(table[b, dst // block_size])
            if 0 <= bs_ < NB and 0 <= bd < NB:
                pool[bd, :, dst % block_size] = pool[bs_, :, src % block_size]
    return new
