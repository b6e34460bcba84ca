"""Plain definitions of the continuous-batching operators, in Python and 64-bit numpy (test infrastructure).

Written from the definitions, one fork, one row, one head at a time; nothing is shared with the CUDA sources.
"""
from __future__ import annotations

import math
from collections import Counter

import numpy as np

REFUSED, BAD = 128, 4


def fork_pages(parents, children, lens, ctx, table, held, free_ids, head, shares, *, block_size, num_blocks):
    B, MB = table.shape
    table, ctx_out, held_out, shares = table.copy(), ctx.copy(), held.copy(), shares.copy()
    F = len(parents)
    named, kin = Counter(int(x) for x in children), {int(x) for x in parents}
    src, dst, granted = np.full(F, -1), np.full(F, -1), np.zeros(F, np.int64)
    head0, promised, status = max(0, int(head)), 0, 0
    head = head0
    for c in range(F):
        p, k = int(parents[c]), int(children[c])
        ok = 0 <= p < B and 0 <= k < B and named[k] == 1 and k not in kin and held[k] <= 0
        L = need = full = 0
        if ok:
            L = max(0, int(ctx[p]))
            if lens is not None:
                L = min(L, max(0, int(lens[c])))
            full, need = L // block_size, int(L % block_size > 0)
            ok = full + need <= min(int(held[p]), MB)
            if not ok:
                need = 0
        promised += need
        if ok and need and head0 + promised > len(free_ids):
            ok = False
        if not ok:
            status |= REFUSED
            continue
        granted[c] = 1
        for j in range(full):
            table[k, j] = table[p, j]
            if 0 <= table[p, j] < num_blocks:
                shares[table[p, j]] += 1
            else:
                status |= BAD
        if need:
            head = head0 + promised
            table[k, full] = free_ids[head - 1]
            if 0 <= table[p, full] < num_blocks and 0 <= table[k, full] < num_blocks:
                src[c], dst[c] = table[p, full], table[k, full]
            else:
                status |= BAD
        ctx_out[k], held_out[k] = L, full + need
    return dict(table=table, ctx=ctx_out, held=held_out, head=head, shares=shares, copy_src=src, copy_dst=dst, granted=granted,
                status=status)


def release_pages(rows, keep, ctx, table, held, free_ids, head, shares, *, block_size, num_blocks):
    B, MB = table.shape
    ctx_out, held_out, shares, free_ids = ctx.copy(), held.copy(), shares.copy(), free_ids.copy()
    status, given, named = 0, [], Counter(int(x) for x in rows)
    for c, r in enumerate(rows):
        r = int(r)
        if not 0 <= r < B or named[r] != 1:
            status |= REFUSED
            continue
        k = 0 if keep is None else max(0, int(keep[c]))
        end = min(max(0, int(held[r])), MB)
        stay = min(end, -(-k // block_size))
        for j in range(stay, end):
            if 0 <= table[r, j] < num_blocks:
                given.append(int(table[r, j]))
            else:
                status |= BAD
        ctx_out[r], held_out[r] = min(max(0, int(ctx[r])), k), stay
    freed, times = [], Counter(given)
    for b in dict.fromkeys(given):           # in the order of their first places
        left = int(shares[b]) - times[b]
        if left < 0:
            freed.append(b)
        shares[b] = max(0, left)
    head = min(max(0, int(head)), len(free_ids))
    put = min(len(freed), head)
    if put < len(freed):
        status |= REFUSED
    free_ids[head - put: head] = freed[:put]
    return dict(free=free_ids, ctx=ctx_out, held=held_out, head=head - put, shares=shares, status=status)


def head_norm(x, weight, eps, offset):
    """x [..., D] in 64 bits, weight [D] or None."""
    y = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    return y if weight is None else y * (weight + offset)


def turn(x, positions, inv_freq, interleaved, magnitude=1.0):
    """Rotary positions of x [T, heads, D] in 64 bits."""
    half = len(inv_freq)
    y = x.copy()
    for t, pos in enumerate(positions):
        for j in range(half):
            a, b = (2 * j, 2 * j + 1) if interleaved else (j, j + half)
            c, s = magnitude * math.cos(float(pos) * float(inv_freq[j])), magnitude * math.sin(float(pos) * float(inv_freq[j]))
            y[t, :, a] = x[t, :, a] * c - x[t, :, b] * s
            y[t, :, b] = x[t, :, b] * c + x[t, :, a] * s
    return y


def chunk_attention(q, k, v, n, scale):
    """q [n, Hq, D], k and v [T, Hkv, D] of one sequence.  Returns (out, sum of weights x |v|, largest sum of |q_d k_d| of a
    row), all [n, Hq, ...]."""
    _, Hq, D = q.shape
    T, Hkv = k.shape[0], k.shape[1]
    out, mag, spread = np.zeros((n, Hq, D)), np.zeros((n, Hq, D)), np.zeros((n, Hq))
    for i in range(n):
        seen = min(T, T - n + i + 1)
        if seen <= 0:
            continue
        for h in range(Hq):
            kk, vv = k[:seen, h // (Hq // Hkv)], v[:seen, h // (Hq // Hkv)]
            s = kk @ q[i, h] * scale
            w = np.exp(s - s.max())
            w /= w.sum()
            out[i, h], mag[i, h] = w @ vv, w @ np.abs(vv)
            spread[i, h] = (np.abs(kk) @ np.abs(q[i, h])).max() * scale
    return out, mag, spread


def shape_logits(x, *, temperature=1.0, repetition=None, frequency=None, presence=None, text=(), prompt=0, branch=(), bias=(),
                 allowed=None):
    """One row: x [V] in 64 bits; text = the history's tokens, the first `prompt` of them the prompt, branch = drafted tokens,
    bias = (token, value) pairs, allowed = truth values [V] or None.  Returns (shaped logits, probabilities)."""
    V = len(x)
    x = np.where(np.isnan(x), -np.inf, x)
    text = [int(t) for t in text]
    if repetition is not None or frequency is not None or presence is not None:
        r = 1.0 if repetition is None or not repetition > 0 else float(repetition)
        f, p = (0.0 if z is None else float(z) for z in (frequency, presence))
        made = {}
        for t in text[prompt:] + [int(t) for t in branch]:
            made[t] = made.get(t, 0) + 1
        for t in set(text) | set(made):
            if 0 <= t < V:
                x[t] = x[t] / r if x[t] > 0 else x[t] * r
                n = made.get(t, 0)
                if n:
                    x[t] = x[t] - f * n - p
    for t, b in bias:
        if 0 <= t < V:
            x[t] += b
    if allowed is not None:
        x = np.where(allowed, x, -np.inf)
    x = np.where(np.isnan(x), -np.inf, x)
    probs = np.zeros(V)
    top = x.max()
    if top == -np.inf:
        return x, probs
    if temperature > 0:
        w = np.where(x == top, 1.0, 0.0)
        rest = (x != top) & (x != -np.inf)
        w[rest] = np.exp((x[rest] - top) / temperature)
        return x, w / w.sum()
    probs[int(np.argmax(x))] = 1.0
    return x, probs
