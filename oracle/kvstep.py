"""KV cache operators of a serving step (oracle): places for new tokens,
rotary positions with the cache write, and attention over the paged cache.

TEST INFRASTRUCTURE ONLY (see oracle/__init__.py).

Sec. III-B names "KV-cache operators with variable-length shards".  Readings:
  * the ids given out are those that no table entry names, ascending, in
    (sequence, block) order; a step that cannot be served whole changes
    nothing;
  * a block that takes new tokens may be named by one entry only;
  * query head h (global) reads KV head h // group (global);
  * a token sees the tokens of its sequence at or before its position,
    inside the window if there is one, whose block is present;
  * everything is computed in 64 bits, entry by entry.
"""
from __future__ import annotations

import math

import numpy as np

OK, EINVAL, ECAPACITY = 0, -1, -2


def extend(table, cached, fresh, block_tokens, num_blocks, max_tokens):
    """-> (table, starts, slots, positions, status)"""
    table = np.asarray(table, dtype=np.int64)
    n, cols = table.shape
    starts, slots, positions = [0] * (n + 1), [-1] * max_tokens, [0] * max_tokens

    def refused(code, wanted=0, free=0):
        return table.copy(), starts, slots, positions, [code, 0, wanted, free]

    total = 0
    for c, f in zip(cached, fresh):
        if c < 0 or f < 0 or c + f > cols * block_tokens:
            return refused(EINVAL)
        total += f
    if total > max_tokens:
        return refused(EINVAL)
    uses = {}
    for p in table.ravel().tolist():
        if p < -1 or p >= num_blocks:
            return refused(EINVAL)
        if p >= 0:
            uses[p] = uses.get(p, 0) + 1
    free = [p for p in range(num_blocks) if p not in uses]
    new, wanted = table.copy(), []
    for s in range(n):
        if not fresh[s]:
            continue
        for b in range(cached[s] // block_tokens, -(-(cached[s] + fresh[s]) // block_tokens)):
            if table[s, b] == -1:
                wanted.append((s, b))
            elif uses[int(table[s, b])] > 1:
                return refused(EINVAL)
    if len(wanted) > len(free):
        return refused(ECAPACITY, len(wanted), len(free))
    for (s, b), p in zip(wanted, free):
        new[s, b] = p
    t = 0
    for s in range(n):
        starts[s] = t
        for i in range(fresh[s]):
            pos = cached[s] + i
            slots[t] = int(new[s, pos // block_tokens]) * block_tokens + pos % block_tokens
            positions[t] = pos
            t += 1
    starts[n] = t
    return new, starts, slots, positions, [OK, total, len(wanted), len(free) - len(wanted)]


def frequencies(rot_dim, base, scaling="plain", factor=1.0, low=0.0, high=0.0, original=0.0):
    """Radians per position of each pair."""
    out = []
    for i in range(rot_dim // 2):
        f = base ** (-2.0 * i / rot_dim)
        if scaling == "linear":
            f = f / factor
        elif scaling == "parts":
            turns = original * f / (2 * math.pi)
            keep = min(1.0, max(0.0, (turns - low) / (high - low)))
            f = f * keep + f / factor * (1 - keep)
        out.append(f)
    return out


def rotate(x, positions, freqs, interleaved=False, amplitude=1.0):
    """x float64 [tokens, heads, head_dim], turned."""
    y = x.copy()
    n = len(freqs)
    for i, f in enumerate(freqs):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + n)
        for t, pos in enumerate(positions):
            angle = float(pos) * f
            c, s = amplitude * math.cos(angle), amplitude * math.sin(angle)
            y[t, :, a] = x[t, :, a] * c - x[t, :, b] * s
            y[t, :, b] = x[t, :, b] * c + x[t, :, a] * s
    return y


def attend(q, keys, values, starts, cached, q_heads, kv_heads, group, scale, softcap=0.0, window=0, slopes=None,
           seen=None):
    """q float64 [tokens, query heads, dim]; keys / values: per sequence float64
    [context, KV heads, dim]; seen: per sequence a truth value per context
    token (False where its block is absent).
    -> out, lse, weight (sum of p |v| over sum of p, per dimension), reach
    (largest sum of |q_d k_d| * scale over the seen tokens, per row and head)"""
    rows, n_q, dim = q.shape
    out, weight = np.zeros((rows, n_q, dim)), np.zeros((rows, n_q, dim))
    lse, reach = np.full((rows, n_q), -np.inf), np.zeros((rows, n_q))
    for s in range(len(starts) - 1):
        for r in range(starts[s], starts[s + 1]):
            pos = cached[s] + r - starts[s]
            first = max(0, pos - window + 1) if window else 0
            at = np.array([t for t in range(first, pos + 1) if seen is None or seen[s][t]], dtype=int)
            if not len(at):
                continue
            for h in range(n_q):
                kh = (q_heads[0] + h) // group - kv_heads[0]
                K, V = keys[s][at, kh], values[s][at, kh]
                z = scale * (K @ q[r, h])
                reach[r, h] = abs(scale) * np.max(np.abs(K) @ np.abs(q[r, h]))
                if softcap:
                    z = softcap * np.tanh(z / softcap)
                if slopes is not None:
                    z = z + slopes[h] * (at - pos)
                top = z.max()
                p = np.exp(z - top)
                total = p.sum()
                out[r, h] = (p[:, None] * V).sum(0) / total
                weight[r, h] = (p[:, None] * np.abs(V)).sum(0) / total
                lse[r, h] = top + math.log(total)
    return out, lse, weight, reach
