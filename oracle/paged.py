"""Serving a batch over a paged cache: block tables and slot maps from request lengths, the write
of keys and values by slot, and attention behind a shared prefix, in plain numpy.

The paper's engine batches requests in flight (Sec. II-C) and says nothing of its tables; the
rules are the library's (include/ftts.h).  Attention is the softmax average over the tokens that
a row sees, in float64.
"""
import numpy as np

PAGE = 64


def build_tables(cached, added, free, n_pages, table, max_rows):
    """(table, row_offsets, seq_lens, slots, counts) as ftts_build_tables defines them."""
    B, width = table.shape
    table = table.copy()
    slots = np.full(max_rows, -1, dtype=np.int64)
    offsets, lens = [0], []
    taken = refused = asked = 0
    for b in range(B):
        c, a = int(cached[b]), int(added[b])
        fits = c >= 0 and a >= 0 and c + a <= width * PAGE
        has = min(-(-max(c, 0) // PAGE), width)
        need = -(-(c + a) // PAGE) if fits else has
        asked += need - has
        ok = fits and (need == has or asked <= len(free))
        table[b, has:] = -1
        if ok:
            table[b, has:need] = free[asked - (need - has):asked]
            if need > has:
                taken = asked
            for i in range(a):
                r, t = offsets[-1] + i, c + i
                page = table[b, t // PAGE]
                if r < max_rows and 0 <= page < n_pages:
                    slots[r] = page * PAGE + t % PAGE
        refused += not ok
        lens.append(c + a if ok else max(c, 0))
        offsets.append(min(offsets[-1] + max(a, 0), 2 ** 31 - 1))
    return table, np.array(offsets), np.array(lens), slots, np.array([taken, refused])


def append(pool, layer, k, v, slots):
    """pool [L][pages][2][H][64][64] with rows k, v [T][H * 64] at their slots (a copy)."""
    pool = pool.copy()
    H = pool.shape[3]
    for r, s in enumerate(slots):
        if 0 <= s < pool.shape[1] * PAGE:
            pool[layer, s // PAGE, 0, :, s % PAGE] = k[r].reshape(H, -1)
            pool[layer, s // PAGE, 1, :, s % PAGE] = v[r].reshape(H, -1)
    return pool


def tokens_seen(n_pages, prefix_pages, prefix_len, table_row, own):
    """(page, slot) of the prefix's tokens and the first `own` of a sequence, without those in pages
    outside the pool."""
    at = [(prefix_pages[t // PAGE], t % PAGE) for t in range(prefix_len)]
    at += [(table_row[t // PAGE], t % PAGE) for t in range(min(own, len(table_row) * PAGE))]
    at = np.array([x for x in at if 0 <= x[0] < n_pages], dtype=np.int64).reshape(-1, 2)
    return at[:, 0], at[:, 1]


def shared_attention(q, pool, prefix_pages, prefix_len, table, seq_lens, row_offsets, weights=False):
    """Rows q [T][n_head][64] over pool [pages][2][n_kv_head][64][64]: out [T][n_head][64], NaN in rows of
    no sequence.  With weights also, per row and head, (sum p |v| / sum p, the largest sum_d |q_d k_d| / 8,
    the number of tokens seen)."""
    T, H, D = q.shape
    G = H // pool.shape[2]
    out = np.full((T, H, D), np.nan)
    size, dots, count = np.zeros((T, H, D)), np.zeros((T, H)), np.zeros(T, dtype=np.int64)
    for b in range(len(seq_lens)):
        r0, r1 = (b, b + 1) if row_offsets is None else (row_offsets[b], row_offsets[b + 1])
        for r in range(r0, r1):
            own = seq_lens[b] - (r1 - r0) + (r - r0) + 1
            pg, sl = tokens_seen(len(pool), prefix_pages, prefix_len, table[b], max(own, 0))
            if seq_lens[b] < 0 or len(pg) == 0:
                out[r] = 0.0
                continue
            count[r] = len(pg)
            for h in range(H):
                k, v = (pool[pg, j, h // G, sl].astype(np.float64) for j in (0, 1))
                s = k @ q[r, h].astype(np.float64) / np.sqrt(D)
                p = np.exp(s - s.max())
                out[r, h] = (p @ v) / p.sum()
                if weights:
                    size[r, h] = (p @ np.abs(v)) / p.sum()
                    dots[r, h] = (np.abs(k) @ np.abs(q[r, h].astype(np.float64))).max() / np.sqrt(D)
    return (out, size, dots, count) if weights else out
