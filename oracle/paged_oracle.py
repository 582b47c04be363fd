"""The paged cache in plain numpy: block tables by loops, summaries and page choice by their definition, attention in 64 bits."""
from __future__ import annotations

import numpy as np

PAGE = 64


def tables(new, past, free, table, n_tokens):
    """free: list of free pages, oldest first.  Returns (table, q_begin, kv_len, slots, positions, pages handed out, refused)."""
    table = table.copy()
    q_begin, kv, slots, positions = [0], [], [], []
    taken = wanted = refused = 0
    for i, (n, p) in enumerate(zip(new, past)):
        n, p = max(int(n), 0), max(int(p), 0)
        had, has = -(-p // PAGE), -(-(p + n) // PAGE)
        ok = has <= table.shape[1]
        if ok and has > had:
            wanted += has - had
            ok = wanted <= len(free)
        if ok:
            for pg in range(had, has):
                table[i, pg] = free[taken]
                taken += 1
        else:
            refused += 1
        kv.append(p + n if ok else 0)
        for pos in range(p, p + n):
            positions.append(pos)
            slots.append(int(table[i, pos // PAGE]) * PAGE + pos % PAGE if ok else -1)
        q_begin.append(q_begin[-1] + n)
    more = n_tokens - len(slots)
    return table, np.array(q_begin), np.array(kv), np.array(slots + [-1] * more), np.array(positions + [0] * more), taken, refused


def _codes(x):
    """float32 [.., d] -> (codes, scale): every step in 32 bits."""
    scale = np.abs(x).max(-1) * (np.float32(1) / np.float32(127))
    safe = np.where(scale > 0, scale, np.float32(1))
    return np.where(scale[..., None] > 0, np.clip(np.rint(x / safe[..., None]), -127, 127), 0).astype(np.int64), scale


def summary(keys):
    """float32 [64, d] -> (codes, scale) of the mean key, summed as a tree by halves."""
    while len(keys) > 1:
        keys = keys[: len(keys) // 2] + keys[len(keys) // 2:]
    return _codes(keys[0] * np.float32(1 / PAGE))


def select(q, codes, scales, pos, sink, local, n_select):
    """q float32 [G, d] of one group, codes [pages, d], scales [pages]: the pages the token at `pos` takes, ascending."""
    total = q[0]
    for g in range(1, len(q)):
        total = total + q[g]
    mine, _ = _codes(total)
    pages = pos // PAGE + 1
    score = (codes[:pages].astype(np.int64) @ mine).astype(np.float32) * scales[:pages].astype(np.float32)
    must = [p for p in range(pages) if p < sink or p >= pages - local]
    rest = sorted((p for p in range(pages) if p not in set(must)), key=lambda p: (-score[p], p))
    return sorted(must + rest[: n_select - len(must)])


def attention(q, k, v, seen, scale):
    """q [rows, d], k, v [keys, d], seen [rows, keys] -> (out, lse, sum of p |v|, sum of |q k| scale per row's largest), 64 bits.
    Keys and values that no row sees take no part, whatever they hold."""
    q, k, v = (np.where(np.isfinite(x), x, 0.0).astype(np.float64) for x in (q, k, v))
    logits = np.where(seen, q @ k.T * scale, -np.inf)
    top = np.max(logits, axis=1, initial=-np.inf, keepdims=True)
    p = np.exp(logits - np.where(np.isfinite(top), top, 0.0))
    total = p.sum(1, keepdims=True)
    p = np.divide(p, total, out=np.zeros_like(p), where=total > 0)
    with np.errstate(divide="ignore"):
        lse = (np.where(np.isfinite(top), top, 0.0) + np.log(total))[:, 0]
    reach = (np.abs(q) @ np.abs(k).T * scale * seen).max(1, initial=0.0)
    return p @ v, lse, p @ np.abs(v), reach
