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


# ---------------------------------------------------------------------------------------------- 4 bits
def _e4m3():
    """The numbers that the 127 bytes 0 .. 126 stand for, ascending."""
    return np.array([m / 512 if e == 0 else (8 + m) * 2.0 ** (e - 10) for e in range(16) for m in range(8)][:127])


def quantise(x, exp=0):
    """Rows [.., d] -> (codes from -7 to 7, scale bytes [.., d / 16])."""
    x = np.asarray(x, dtype=np.float64).reshape(*x.shape[:-1], x.shape[-1] // 16, 16) * 2.0 ** -exp
    want = np.minimum(np.abs(x).max(-1).astype(np.float32) * np.float32(1 / 7), np.float32(448)).astype(np.float64)
    numbers = _e4m3()
    above = np.minimum(np.searchsorted(numbers, want), 126)
    below = np.maximum(above - 1, 0)
    up, down = numbers[above] - want, want - numbers[below]
    byte = np.where(up < down, above, np.where(up > down, below, np.where(above % 2 == 0, above, below)))
    scale = numbers[byte][..., None]
    code = np.where(scale > 0, np.clip(np.rint(x / np.where(scale > 0, scale, 1.0)), -7, 7), 0)
    return code.reshape(*x.shape[:-2], 16 * x.shape[-2]).astype(np.int64), byte.astype(np.int64)


def values(code, byte, exp=0):
    """What codes and scale bytes stand for."""
    return (code.reshape(*byte.shape, 16) * _e4m3()[byte][..., None]).reshape(code.shape) * 2.0 ** exp


def block(k, v):
    """64 rows of K and V as (codes [64, d], bytes [64, d / 16]) -> the bytes of a page of one head."""
    out = []
    for code, _ in (k, v):
        for row in code + 8:
            for c in range(0, len(row), 8):
                fields = [*row[c: c + 8: 2], *row[c + 1: c + 8: 2]]
                word = sum(int(f) << (4 * i) for i, f in enumerate(fields))
                out += [word >> (8 * i) & 255 for i in range(4)]
    return np.array(out + [int(b) for _, byte in (k, v) for b in byte.reshape(-1)], dtype=np.uint8)


def unblock(data, d):
    """The reverse, of blocks [.., bytes]: two pairs of (codes [.., 64, d], bytes [.., 64, d / 16])."""
    out = []
    for part in range(2):
        at = part * PAGE * d // 2
        quad = data[..., at: at + PAGE * d // 2].reshape(*data.shape[:-1], PAGE, d // 8, 4).astype(np.int64)
        word = quad[..., 0] | quad[..., 1] << 8 | quad[..., 2] << 16 | quad[..., 3] << 24
        code = np.stack([(word >> (4 * (i // 2 + (i % 2) * 4)) & 15) - 8 for i in range(8)], -1).reshape(*word.shape[:-1], d)
        at = PAGE * d + part * PAGE * d // 16
        out.append((code, data[..., at: at + PAGE * d // 16].reshape(*data.shape[:-1], PAGE, d // 16).astype(np.int64)))
    return out


# ---------------------------------------------------------------------------------------------- rows between steps
def _listed(lengths, table):
    return {int(table[i][j]) for i, n in enumerate(lengths) for j in range(-(-n // PAGE))}


def _rows(tables, width):
    return np.array([row + [-1] * (width - len(row)) for row in tables])


def fork(parents, keep, lengths, table, free):
    """free: list of free pages, oldest first.  Returns (lengths, table, moves from, moves to, pages taken, rows cut, pages given back)."""
    n = len(lengths)
    lengths = [max(int(x), 0) for x in lengths]
    on = [0 <= p < n for p in parents]
    new = [min(lengths[p], max(int(k), 0)) if o else 0 for p, k, o in zip(parents, keep, on)]
    listed = _listed(new, [table[p] if o else [] for p, o in zip(parents, on)])
    whole = {int(table[p][j]) for p, m in zip(parents, new) for j in range(m // PAGE)}
    owner = {}
    for i in sorted(range(n), key=lambda i: (parents[i] != i, i)):
        if new[i] % PAGE:
            owner.setdefault(int(table[parents[i]][new[i] // PAGE]), i)
    tables, source, target, taken, cut = [], [], [], 0, 0
    for i in range(n):
        row = [int(x) for x in table[parents[i]][: -(-new[i] // PAGE)]] if on[i] else []
        moves = [(-1, -1)] * PAGE
        if new[i] % PAGE and (row[-1] in whole or owner[row[-1]] != i):
            page = row.pop()
            if taken < len(free):
                row.append(free[taken])
                taken += 1
                for r in range(new[i] % PAGE):
                    moves[r] = (page * PAGE + r, row[-1] * PAGE + r)
            else:
                new[i] = new[i] // PAGE * PAGE
                cut += 1
        tables.append(row)
        source += [a for a, _ in moves]
        target += [b for _, b in moves]
    return np.array(new), _rows(tables, table.shape[1]), np.array(source), np.array(target), taken, cut, sorted(_listed(lengths, table) - listed)


def compact(stays, lengths, table, free, n_moves):
    """stays: truth values [rows][width]; results as `fork`'s, with the rows left as they are in the place of rows cut."""
    lengths = [max(int(x), 0) for x in lengths]
    new, tables, moves, taken, wanted, entries, refused = [], [], [], 0, 0, 0, 0
    listed = set()
    for i, n in enumerate(lengths):
        row = [int(x) for x in table[i][: -(-n // PAGE)]]
        leaves = [t for t in range(min(n, len(stays[i]))) if not stays[i][t]]
        if leaves:
            first = leaves[0] // PAGE
            gone = set(leaves)
            staying = [t for t in range(first * PAGE, n) if t not in gone]
            need = -(-len(staying) // PAGE)
            wanted += need
            entries += len(staying)
            if need == 0 or (wanted <= len(free) and entries <= n_moves):
                old, row = row, row[:first] + list(free[taken: taken + need])
                listed |= set(old[:first])
                taken += need
                moves += [(old[t // PAGE] * PAGE + t % PAGE, row[first + k // PAGE] * PAGE + k % PAGE) for k, t in enumerate(staying)]
                n = first * PAGE + len(staying)
            else:
                refused += 1
                listed |= set(row)
        else:
            listed |= set(row)
        new.append(n)
        tables.append(row)
    done = len(moves)
    moves += [(-1, -1)] * (n_moves - done)
    back = sorted(_listed(lengths, table) - listed)
    return np.array(new), _rows(tables, table.shape[1]), np.array([a for a, _ in moves]), np.array([b for _, b in moves]), taken, refused, back, done
