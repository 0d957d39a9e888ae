"""Checking drafted trees over a paged cache: rows turned by their positions, attention of a tree of
drafted tokens and the commit of its accepted path, in plain numpy (float64).

The paper's engine generates token by token (Sec. II-C) and says nothing of drafts; the rules are the
library's (include/ftts.h).
"""
import math

import numpy as np

PAGE = 64
HALVES, PAIRS = 0, 1
PLAIN, LINEAR, BASE, PARTS = 0, 1, 2, 3


def frequencies(dim, base, scaling=PLAIN, factor=1.0, original=1024.0, slow=1.0, fast=32.0):
    """(radians a position of each pair, factor of the turned columns)."""
    if scaling == BASE:
        base = base * factor ** (dim / (dim - 2))
    f = base ** (-np.arange(0, dim, 2, dtype=np.float64) / dim)
    if scaling == LINEAR:
        f = f / factor
    if scaling == PARTS:
        turns = original * f / (2 * math.pi)
        stay = np.clip((turns - slow) / (fast - slow), 0, 1)
        f = stay * f + (1 - stay) * f / factor
    return f, 0.1 * math.log(factor) + 1 if scaling == PARTS else 1.0


def rotate(x, positions, dim, layout, freq, scale=1.0):
    """Rows x [T][heads * 64] turned by their positions."""
    y = x.astype(np.float64).reshape(len(x), -1, 64).copy()
    h = dim // 2
    unit = scale * np.exp(1j * positions.astype(np.float64)[:, None] * freq)[:, None]
    a, b = (slice(0, h), slice(h, dim)) if layout == HALVES else (slice(0, dim, 2), slice(1, dim, 2))
    z = (y[..., a] + 1j * y[..., b]) * unit
    y[..., a], y[..., b] = z.real, z.imag
    return y.reshape(x.shape)


def masks(parents, words):
    """[n][words] bits of each token's ancestors and itself, as int64."""
    seen = []
    for i, p in enumerate(parents):
        seen.append((seen[p] if 0 <= p < i else 0) | 1 << i)
    return np.array([[m >> 64 * w & (1 << 64) - 1 for w in range(words)] for m in seen], dtype=np.uint64).view(np.int64)


def depths(parents):
    out = []
    for p in parents:
        out.append(out[p] + 1 if p >= 0 else 0)
    return np.array(out)


def attention(q, pool, prefix_pages, prefix_len, table, seq_lens, row_offsets, words, weights=False):
    """Rows q [T][n_head][64] over pool [pages][2][n_kv_head][64][64]: out [T][n_head][64], NaN in rows of no
    sequence.  Row i of a sequence sees the prefix, its own tokens before the tree, and the tree's tokens whose bits
    words[row] has.  With weights also, per row and head, (sum p |v| / sum p, the largest sum_d |q_d k_d| / 8, the
    number of tokens seen)."""
    T, H, D = q.shape
    G = H // pool.shape[2]
    out = np.full((T, H, D), np.nan)
    size, dots, count = np.zeros((T, H, D)), np.zeros((T, H)), np.zeros(T, dtype=np.int64)
    bits = words.view(np.uint64)
    for b in range(len(seq_lens)):
        r0, r1 = row_offsets[b], row_offsets[b + 1]
        past = int(seq_lens[b]) - (r1 - r0)
        for r in range(r0, r1):
            if past < 0:
                out[r] = 0.0
                continue
            own = list(range(past))
            own += [past + j for j in range(min(r1 - r0, 64 * words.shape[1])) if int(bits[r, j // 64]) >> (j % 64) & 1]
            at = [(prefix_pages[t // PAGE], t % PAGE) for t in range(prefix_len)]
            at += [(table[b][t // PAGE], t % PAGE) for t in own if t < len(table[b]) * PAGE]
            at = np.array([x for x in at if 0 <= x[0] < len(pool)], dtype=np.int64).reshape(-1, 2)
            if len(at) == 0:
                out[r] = 0.0
                continue
            count[r] = len(at)
            for h in range(H):
                k, v = (pool[at[:, 0], j, h // G, at[:, 1]].astype(np.float64) for j in (0, 1))
                s = k @ q[r, h].astype(np.float64) / np.sqrt(D)
                p = np.exp(s - s.max())
                out[r, h] = (p @ v) / p.sum()
                if weights:
                    size[r, h] = (p @ np.abs(v)) / p.sum()
                    dots[r, h] = (np.abs(k) @ np.abs(q[r, h].astype(np.float64))).max() / np.sqrt(D)
    return (out, size, dots, count) if weights else out


def accept(tokens, parents, choices, most):
    """(path, next token) of one tree: from its first token on to the first child that is what the model chose."""
    path = [0]
    while len(path) < most:
        c = choices[path[-1]]
        below = [j for j in range(path[-1] + 1, len(tokens)) if parents[j] == path[-1] and tokens[j] == c and c >= 0]
        if not below:
            break
        path.append(below[0])
    return path, int(choices[path[-1]])


def commit(tokens, parents, choices, row_offsets, table, seq_lens, pool, most, limit=256):
    """(path, counts, next tokens, new lengths, pool) as ftts_tree_commit defines them; pool [L][pages][2][H][64][64]."""
    pool, B = pool.copy(), len(seq_lens)
    path, counts = np.full((B, most), -1), np.zeros(B, dtype=np.int64)
    chosen, lens = np.full(B, -1), np.array(seq_lens).copy()
    for b in range(B):
        r0, r1 = row_offsets[b], row_offsets[b + 1]
        past = int(seq_lens[b]) - (r1 - r0)
        if r1 == r0 or past < 0:
            continue
        r1 = min(r1, r0 + limit)
        p, chosen[b] = accept(tokens[r0:r1], parents[r0:r1], choices[r0:r1], most)
        path[b, :len(p)], counts[b], lens[b] = p, len(p), past + len(p)

        def place(t):
            page = table[b][t // PAGE] if t // PAGE < len(table[b]) else -1
            return (page, t % PAGE) if 0 <= page < pool.shape[1] else None
        old = [None if place(past + j) is None else pool[(slice(None), place(past + j)[0], slice(None), slice(None), place(past + j)[1])].copy()
               for j in p]
        for i, x in enumerate(old):
            to = place(past + i)
            if x is not None and to is not None:
                pool[:, to[0], :, :, to[1]] = x
    return path, counts, chosen, lens, pool

