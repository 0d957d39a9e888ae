"""Performance cases of the operators that check drafted trees over the paged cache: rows turned by
their positions, keys and values turned on their way into pages, attention of a tree of drafted
tokens over its sequence's pages, and the commit of the accepted path.

``listed()`` holds the fixed cases, ``draw`` makes more of the same ranges.  Where ``own``
is true ``run`` calls the package; otherwise it computes the same outputs in their plain
form, elementary torch operations in fp32 (angles in fp64: a position of a million times a
frequency leaves no fraction in fp32).  ``exact`` follows the definitions in float64.

Sizes: heads of 64 wide and pages of 64 tokens, as everywhere in this package; 20 and 12
heads are its two models', 24 layers and a vocabulary of 8194 its large one's.  Queries, keys
and values are drawn at the spread a LayerNorm output through a 1280-wide N(0, 0.02) linear
has, N(0, 0.7).
"""
import math
import random

import torch

own = False
DEV, PAGE, DIM, VOCAB = "cuda", 64, 64, 8194
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---- the cases -----------------------------------------------------------------------------
def listed():
    return [
        # The queries of one decode step of a server's 32 slots: latency.
        rotate("rotate_step_32", "bf16", "bf16", 32, 20, "halves", 64, 1500),
        # Half of each head turned, neighbours as pairs, for the packed rows of 32 prefixes.
        rotate("rotate_prompt_9746", "bf16", "bf16", 9746, 20, "pairs", 32, 512, packed=True),
        # One utterance's tree of 12 drafted tokens: the fp32 projection into a bf16 cache.
        append("append_tree_12", "f32", "bf16", 12, 20, 20, "halves", 64, 700, packed=True),
        # A server's trees on a model whose five query heads share a key head, padded as a captured call is.
        append("append_trees_1024_grouped", "bf16", "bf16", 1024, 20, 4, "pairs", 64, 2000, pad=41, packed=True),
        # Packed prompts far into a context that was stretched eightfold.
        append("append_prompt_10827_far", "bf16", "bf16", 10827, 20, 20, "halves", 64, 32000, pad=173, packed=True,
               base=500000.0, scaling="parts", factor=8.0, original=4096),
        # One utterance's tree of 16 drafted tokens early in the utterance: latency.
        tree("tree_1", "bf16", 1, 20, 20, 0, 300, 300, 16, 16),
        # A server's slots in mid-utterance, trees of 8 to 64 tokens.
        tree("tree_32", "bf16", 32, 20, 20, 0, 64, 1200, 8, 64),
        # Grouped heads behind a prefix that the batch shares.
        tree("tree_16_grouped", "bf16", 16, 20, 4, 1500, 0, 1200, 12, 48),
        # A few long contexts, wide trees: reading and products alike.
        tree("tree_4_long", "bf16", 4, 20, 20, 0, 6000, 14000, 40, 64),
        # The fp32 mode's cache, a few utterances.
        tree("tree_4_f32", "f32", 4, 20, 20, 0, 50, 700, 8, 32),
        # One utterance's step: four of 16 tokens are kept, in all 24 layers.
        commit("commit_1", "bf16", 1, 24, 20, 20, 150, 16, 16, 4, 4),
        # A server's slots, one to eight tokens kept of each tree.
        commit("commit_16", "bf16", 16, 24, 20, 20, 150, 16, 64, 1, 8),
    ]


def _turn(layout, dim, base, scaling, factor, original):
    return {"layout": layout, "dim": dim, "base": base, "scaling": scaling, "factor": factor, "original": original}


def rotate(name, src, dst, rows, heads, layout, dim, far, packed=False, base=10000.0, scaling="plain", factor=1.0,
           original=1024):
    """`rows` rows at positions up to `far`; packed: they are columns of q/k/v rows."""
    return {"name": name, "kind": "rotate", "src": src, "dst": dst, "rows": rows, "heads": heads, "far": far,
            "packed": packed, **_turn(layout, dim, base, scaling, factor, original)}


def append(name, src, dst, rows, heads, kv_heads, layout, dim, far, pad=0, packed=False, base=10000.0, scaling="plain",
           factor=1.0, original=1024):
    """`rows` new tokens and `pad` rows without a slot; packed: q, k and v are columns of one row."""
    return {"name": name, "kind": "append", "src": src, "dst": dst, "rows": rows, "heads": heads, "kv_heads": kv_heads,
            "far": far, "pad": pad, "packed": packed, **_turn(layout, dim, base, scaling, factor, original)}


def tree(name, dtype, batch, heads, kv_heads, prefix, past_lo, past_hi, lo, hi, lens_seed=3):
    """Trees of lo to hi tokens, own tokens cached before them in [past_lo, past_hi], behind `prefix` shared ones."""
    return {"name": name, "kind": "tree", "dtype": dtype, "batch": batch, "heads": heads, "kv_heads": kv_heads,
            "prefix": prefix, "past_lo": past_lo, "past_hi": past_hi, "lo": lo, "hi": hi, "lens_seed": lens_seed}


def commit(name, dtype, batch, layers, kv_heads, past_lo, past_hi, lo, hi, keep_lo, keep_hi, lens_seed=3):
    """Trees of lo to hi tokens of which keep_lo to keep_hi are kept (the first always)."""
    return {"name": name, "kind": "commit", "dtype": dtype, "batch": batch, "layers": layers, "kv_heads": kv_heads,
            "past_lo": past_lo, "past_hi": past_hi, "lo": lo, "hi": hi, "keep_lo": keep_lo, "keep_hi": keep_hi,
            "lens_seed": lens_seed}


def draw(rng):
    def log_int(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    def span(lo, hi):
        a, b = log_int(lo + 1, hi + 1) - 1, log_int(lo + 1, hi + 1) - 1
        return min(a, b), max(a, b)

    kind = rng.choices(["rotate", "append", "tree", "commit"], [2, 3, 6, 2])[0]
    if kind in ("rotate", "append"):
        src, dst = rng.choice([("bf16", "bf16"), ("bf16", "bf16"), ("f32", "bf16"), ("f32", "f32")])
        rows = log_int(1, 4000 if src == "f32" else 10000)
        turn = {"base": rng.choice([10000.0, 500000.0]), "packed": rng.random() < 0.6,
                **rng.choice([{}, {"scaling": "linear", "factor": 4.0}, {"scaling": "parts", "factor": 8.0, "original": 4096}])}
        layout, dim = rng.choice(["halves", "pairs"]), rng.choice([64, 64, 32, 16, 48, 24, 2 * rng.randint(1, 32)])
        far = log_int(rows, 1 << 20)
        if kind == "rotate":
            c = rotate("", src, dst, rows, rng.choice([20, 12, 4, 1]), layout, dim, far, **turn)
        else:
            heads, kv_heads = rng.choice([(20, 20), (20, 20), (12, 12), (20, 4), (12, 2), (8, 1)])
            c = append("", src, dst, rows, heads, kv_heads, layout, dim, far, rng.choice([0, rng.randrange(64)]), **turn)
    elif kind == "tree":
        dtype = rng.choices(["bf16", "f32"], [4, 1])[0]
        heads, kv_heads = rng.choice([(20, 20), (20, 20), (12, 12), (4, 4), (20, 4), (12, 2), (8, 1)])
        batch, (lo, hi) = log_int(1, 64), span(1, 256)
        lo, hi = max(1, lo), max(1, hi)
        past = span(0, rng.choice([1200, 1200, 14000]))
        prefix = rng.choice([0, 0, log_int(1, 6000)])
        # no more scores than the largest listed case has
        most = max(1, (4000000 if dtype == "f32" else 60000000) // (heads * hi))
        batch = max(1, min(batch, most // 1500))
        prefix = min(prefix, most // (2 * batch))
        past = tuple(min(p, max(0, most // batch - prefix)) for p in past)
        c = tree("", dtype, batch, heads, kv_heads, prefix, *past, lo, hi, rng.randrange(1 << 20))
    else:
        layers, kv_heads = rng.choice([(24, 20), (24, 20), (24, 4), (2, 4), (12, 12)])
        lo, hi = span(1, 128)
        lo, hi = max(1, lo), max(1, hi)
        keep = sorted(rng.randint(1, 12) for _ in range(2))
        c = commit("", rng.choice(["bf16", "bf16", "f32"]), log_int(1, 12), layers, kv_heads, *span(0, 150), lo, hi, *keep,
                   rng.randrange(1 << 20))
    del c["name"]
    return c


def _lens(case):
    """(own tokens before the tree, tokens of the tree, tokens kept) of each sequence."""
    r = random.Random(case["lens_seed"])
    n = range(case["batch"])
    past, rows = [r.randint(case["past_lo"], case["past_hi"]) for _ in n], [r.randint(case["lo"], case["hi"]) for _ in n]
    return past, rows, [min(r.randint(case.get("keep_lo", 1), case.get("keep_hi", 1)), (m + 1) // 2) for m in rows]


def _pages(tokens):
    return -(-tokens // PAGE)


def _frequencies(case):
    """Radians a position of each pair, and the factor of the turned columns."""
    f = [case["base"] ** (-2.0 * i / case["dim"]) for i in range(case["dim"] // 2)]
    if case["scaling"] == "linear":
        return [x / case["factor"] for x in f], 1.0
    if case["scaling"] == "parts":
        # pairs that turn 32 times and more within the original length stay, those of a turn or less are stretched
        out = []
        for x in f:
            keep = min(max((case["original"] * x / (2 * math.pi) - 1.0) / 31.0, 0.0), 1.0)
            out.append(x * keep + x / case["factor"] * (1 - keep))
        return out, 0.1 * math.log(case["factor"]) + 1.0
    return f, 1.0


# ---- inputs ----------------------------------------------------------------------------------
def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) + 77)
    order = random.Random(int(seed))
    return {"rotate": _prepare_rotate, "append": _prepare_append, "tree": _prepare_tree,
            "commit": _prepare_commit}[case["kind"]](case, order, g)


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _normal(shape, g, dtype):
    return torch.randn(shape, generator=g, device=DEV).mul_(0.7).to(TYPES[dtype])


def _with_rotary(case, s):
    f, s["scale"] = _frequencies(case)
    s["freq"], s["layout"], s["dim"] = torch.tensor(f, dtype=torch.float64, device=DEV), case["layout"], case["dim"]
    if own:
        # the rotation that a program describes once
        from paper_2607_21042_amd import ftts
        layout = {"halves": ftts.ROTARY_HALVES, "pairs": ftts.ROTARY_PAIRS}[case["layout"]]
        scaling = {"plain": ftts.ROTARY_PLAIN, "linear": ftts.ROTARY_LINEAR, "parts": ftts.ROTARY_PARTS}[case["scaling"]]
        s["rotary"] = ftts.Rotary(case["dim"], layout, case["base"], scaling, case["factor"], case["original"])
    return s


def _runs(rows, far, order):
    """Positions of `rows` tokens: runs of neighbours, the last one at `far` at most."""
    out = []
    while len(out) < rows:
        n = min(rows - len(out), order.randint(1, 512))
        first = order.randint(0, max(0, far - n))
        out += range(first, first + n)
    return out


def _prepare_rotate(case, order, g):
    T, width = case["rows"], case["heads"] * DIM
    x = _normal((T, (3 if case["packed"] else 1) * width), g, case["src"])[:, :width]
    return _with_rotary(case, {"kind": "rotate", "x": x, "positions": _i32(_runs(T, case["far"], order)),
                               "out": torch.zeros((T, width), dtype=TYPES[case["dst"]], device=DEV)})


def _prepare_append(case, order, g):
    T, H, KH = case["rows"], case["heads"], case["kv_heads"]
    n, a, b = T + case["pad"], H * DIM, KH * DIM
    if case["packed"]:
        x = _normal((n, a + 2 * b), g, case["src"])
        q, k, v = x[:, :a], x[:, a:a + b], x[:, a + b:]
    else:
        q, k, v = (_normal((n, w), g, case["src"]) for w in (a, b, b))
    # runs of consecutive slots, one per sequence, in pages of any order
    pages = _pages(T) + 3
    ids = order.sample(range(pages), pages)
    at = order.randrange(PAGE)
    slots = [ids[(at + i) // PAGE] * PAGE + (at + i) % PAGE for i in range(T)] + [-1] * case["pad"]
    dst = TYPES[case["dst"]]
    s = {"kind": "append", "q": q, "k": k, "v": v, "slots": _i32(slots), "heads": H, "kv_heads": KH,
         "positions": _i32(_runs(n, case["far"], order)), "q_out": torch.zeros((n, a), dtype=dst, device=DEV),
         "pool": torch.zeros((1, pages, 2, KH, PAGE, DIM), dtype=dst, device=DEV)}
    if own:
        # the view of the pool that a program keeps
        from paper_2607_21042_amd import ftts
        s["kv"] = ftts.KVCache.over(s["pool"])
    return _with_rotary(case, s)


def _parents(n, kept, order):
    """A tree of n tokens, parents before children, and a path of `kept` tokens in it whose second is at `kept` or
    behind: moved together, no token lands on another of the path, so that a pass can be repeated on its cache."""
    path = [0] + sorted(order.sample(range(kept, n), kept - 1))
    parents = [-1] + [order.randrange(max(0, i - 12), i) for i in range(1, n)]
    for p, c in zip(path, path[1:]):
        parents[c] = p
    return parents, path


def _masks(parents, words):
    """The bits of each token's ancestors and itself, in `words` words of 64."""
    seen = []
    for i, p in enumerate(parents):
        seen.append((seen[p] if p >= 0 else 0) | 1 << i)
    return [[((m >> 64 * w & (1 << 64) - 1) ^ (1 << 63)) - (1 << 63) for w in range(words)] for m in seen]


def _prepare_tables(lens, order, first, n_pages):
    ids = order.sample(range(n_pages), n_pages)
    table = torch.full((len(lens), max(_pages(n) for n in lens)), -1, dtype=torch.int32)
    k = first
    for b, n in enumerate(lens):
        table[b, :_pages(n)] = torch.tensor(ids[k:k + _pages(n)], dtype=torch.int32)
        k += _pages(n)
    return ids[:first], table.to(DEV)


def _prepare_tree(case, order, g):
    H, KH, P = case["heads"], case["kv_heads"], case["prefix"]
    past, rows, kept = _lens(case)
    lens = [p + n for p, n in zip(past, rows)]
    total = _pages(P) + sum(_pages(n) for n in lens)
    shared, table = _prepare_tables(lens, order, _pages(P), total)
    words, T = _pages(max(rows)), sum(rows)
    masks = [m for n, k in zip(rows, kept) for m in _masks(_parents(n, k, order)[0], words)]
    s = {"kind": "tree", "q": _normal((T, H * DIM), g, case["dtype"]), "pool": _normal((1, total, 2, KH, PAGE, DIM), g, case["dtype"]),
         "table": table, "seq_lens": _i32(lens), "prefix": P, "prefix_pages": _i32(shared), "heads": H, "kv_heads": KH,
         "masks": torch.tensor(masks, dtype=torch.int64, device=DEV), "cu": _i32([sum(rows[:b]) for b in range(len(rows) + 1)]),
         "most_rows": max(rows)}
    if own:
        # what a program keeps: the views of pool, table and prefix, the workspace and the output rows
        from paper_2607_21042_amd import ftts
        s["kv"], s["pt"] = ftts.KVCache.over(s["pool"]), ftts.PageTableView(s["table"], s["seq_lens"])
        s["shared"] = ftts.SharedPrefix(s["prefix_pages"], P) if P else None
        s["ws"] = torch.empty(ftts.tree_attention_workspace_bytes(H, KH, s["kv"].dtype, case["batch"], T, P,
                                                                  s["pt"].c.max_pages), dtype=torch.uint8, device=DEV)
        s["out"] = torch.empty((T, H * DIM), dtype=TYPES[case["dtype"]], device=DEV)
    return s


def _prepare_commit(case, order, g):
    past, rows, kept = _lens(case)
    lens = [p + n for p, n in zip(past, rows)]
    total = sum(_pages(n) for n in lens)
    _, table = _prepare_tables(lens, order, 0, total)
    parents, tokens, choices = [], [], []
    for n, k in zip(rows, kept):
        up, path = _parents(n, k, order)
        ids = order.sample(range(VOCAB), 2 * n)  # drafted tokens, and others that the model chose
        pick = ids[n:]
        for p, c in zip(path, path[1:]):
            pick[p] = ids[c]
        parents, tokens, choices = parents + up, tokens + ids[:n], choices + pick
    B, most = case["batch"], case.get("keep_hi") + 1
    s = {"kind": "commit", "parents": _i32(parents), "tokens": _i32(tokens), "choices": _i32(choices), "table": table,
         "cu": _i32([sum(rows[:b]) for b in range(B + 1)]), "seq_lens": _i32(lens), "most_rows": max(rows),
         "pool": _normal((case["layers"], total, 2, case["kv_heads"], PAGE, DIM), g, case["dtype"]),
         "path": torch.zeros((B, most), dtype=torch.int32, device=DEV), "counts": _i32([0] * B), "next": _i32([0] * B),
         "new_lens": _i32([0] * B)}
    if own:
        # the views that a program keeps
        from paper_2607_21042_amd import ftts
        s["kv"], s["pt"] = ftts.KVCache.over(s["pool"]), ftts.PageTableView(s["table"], s["seq_lens"])
    return s


# ---- one pass --------------------------------------------------------------------------------
def run(s):
    if own:
        from paper_2607_21042_amd import ftts
        if s["kind"] == "rotate":
            ftts.rotate(s["x"], s["rotary"], s["positions"], s["out"])
            return s["out"]
        if s["kind"] == "append":
            ftts.append_rotated(s["k"], s["v"], s["rotary"], s["positions"], s["slots"], s["kv"], 0, q=s["q"], q_out=s["q_out"])
            return {"pool": s["pool"], "q_out": s["q_out"]}
        if s["kind"] == "tree":
            ftts.tree_attention(s["q"], s["kv"], 0, s["pt"], s["masks"], s["cu"], s["out"], s["ws"], prefix=s["shared"])
            return s["out"]
        ftts.tree_commit(s["tokens"], s["parents"], s["choices"], s["cu"], s["pt"], s["kv"], s["path"], s["counts"], s["next"],
                         s["new_lens"])
        return {k: s[k] for k in ("path", "counts", "next", "new_lens", "pool")}
    return {"rotate": _plain_rotate, "append": _plain_append, "tree": _plain_tree, "commit": _plain_commit}[s["kind"]](s)


def _turned(s, x, heads):
    """Rows x [T][heads * 64] turned by their positions, in fp32."""
    a = s["positions"].double()[:, None] * s["freq"]
    c, n, h = a.cos().float()[:, None] * s["scale"], a.sin().float()[:, None] * s["scale"], s["dim"] // 2
    x = x.float().unflatten(1, (heads, DIM))
    turn, rest = x[..., :2 * h], x[..., 2 * h:]
    if s["layout"] == "halves":
        u, w = turn[..., :h], turn[..., h:]
        y = torch.cat([u * c - w * n, w * c + u * n], -1)
    else:
        u, w = turn[..., 0::2], turn[..., 1::2]
        y = torch.stack([u * c - w * n, w * c + u * n], -1).flatten(-2)
    return torch.cat([y, rest], -1).flatten(1)


def _plain_rotate(s):
    return _turned(s, s["x"], s["x"].shape[1] // DIM).to(s["out"].dtype)


def _plain_append(s):
    pool, KH = s["pool"], s["kv_heads"]
    pages, slots = pool.shape[1], s["slots"].long()
    # the row that each slot takes, or none (rows without a slot meet in one behind the last)
    row = torch.full((pages * PAGE + 1,), -1, dtype=torch.long, device=DEV)
    row[torch.where(slots < 0, pages * PAGE, slots)] = torch.arange(slots.numel(), device=DEV)
    row = row[:-1]
    kv = torch.stack([_turned(s, s["k"], KH), s["v"].float()], 1).unflatten(2, (KH, DIM))[row.clamp(min=0)]  # [slot][2][H][64]
    kv = kv.unflatten(0, (pages, PAGE)).permute(0, 2, 3, 1, 4).to(pool.dtype)
    pool[0] = torch.where((row >= 0).view(pages, 1, 1, PAGE, 1), kv, pool[0])
    q = _turned(s, s["q"], s["heads"]).to(s["q_out"].dtype)
    s["q_out"].copy_(torch.where((slots >= 0)[:, None], q, s["q_out"]))
    return {"pool": pool, "q_out": s["q_out"]}


def _plain_tree(s):
    q, pool, KH, P, n = s["q"], s["pool"][0].float(), s["kv_heads"], s["prefix"], s["most_rows"]
    B, T, G, cu = s["table"].shape[0], q.shape[0], s["heads"] // KH, s["cu"].long()
    i = torch.arange(n, device=DEV)
    rows = (cu[:-1, None] + i).clamp(max=T - 1)                                                       # [B][n]
    qb = q.float()[rows].view(B, n, KH, G, DIM).permute(0, 2, 3, 1, 4)                                # [B][KH][G][n][64]
    kp = pool[s["prefix_pages"].long()].permute(1, 2, 0, 3, 4).flatten(2, 3)[:, :, :P]                # [2][KH][P][64]
    ko = pool[s["table"].long().clamp(min=0)].permute(2, 0, 3, 1, 4, 5).flatten(3, 4)                 # [2][B][KH][L][64]
    sp = qb.permute(1, 0, 2, 3, 4).flatten(1, 3).matmul(kp[0].transpose(1, 2).contiguous()) / 8       # [KH][B G n][P]
    so = qb.flatten(2, 3).matmul(ko[0].transpose(2, 3).contiguous()).view(B, KH, G, n, -1) / 8        # [B][KH][G][n][L]
    bits = ((s["masks"][:, :, None] >> torch.arange(64, device=DEV)) & 1).flatten(1).bool()           # [T][64 words]
    count = cu[1:] - cu[:-1]
    node = torch.arange(so.shape[-1], device=DEV) - (s["seq_lens"].long() - count)[:, None]           # [B][L]
    in_tree = (node >= 0) & (node < count[:, None])
    seen = bits[rows].gather(2, node.clamp(0, bits.shape[1] - 1)[:, None].expand(B, n, -1))           # [B][n][L]
    seen = (seen & in_tree[:, None]) | (node < 0)[:, None]
    so = so.masked_fill(~seen[:, None, None], -math.inf)
    sp = sp.view(KH, B, G, n, P).permute(1, 0, 2, 3, 4)
    m = torch.cat([sp, so], -1).amax(-1, keepdim=True)
    sp, so = torch.exp(sp - m), torch.exp(so - m)
    o = sp.permute(1, 0, 2, 3, 4).flatten(1, 3).matmul(kp[1]).view(KH, B, G, n, DIM).permute(1, 0, 2, 3, 4)
    o = o + so.flatten(2, 3).matmul(ko[1]).view(B, KH, G, n, DIM)
    o = o / (sp.sum(-1, keepdim=True) + so.sum(-1, keepdim=True))
    row = torch.arange(T, device=DEV)
    b = torch.searchsorted(cu, row, right=True) - 1
    return o[b, :, :, row - cu[b]].reshape(T, -1).to(q.dtype)


def _plain_commit(s):
    cu, lens, pool, table = s["cu"].long(), s["seq_lens"].long(), s["pool"], s["table"].long()
    B, most, T = cu.numel() - 1, s["path"].shape[1], s["tokens"].numel()
    count = cu[1:] - cu[:-1]
    j = torch.arange(s["most_rows"], device=DEV)
    at = (cu[:-1, None] + j).clamp(max=T - 1)                                                         # [B][n]
    token, parent, real = s["tokens"].long()[at], s["parents"].long()[at], j < count[:, None]
    cur, on = torch.zeros_like(count), count > 0
    path, chosen = [], torch.full_like(count, -1)
    for step in range(most):
        path.append(torch.where(on, cur, -1))
        pick = s["choices"].long()[(cu[:-1] + cur).clamp(max=T - 1)]
        match = (parent == cur[:, None]) & (token == pick[:, None]) & (pick >= 0)[:, None] & real & (j > cur[:, None])
        child = torch.where(match, j, 1 << 30).amin(1)
        stop = on & ((child == 1 << 30) | (step == most - 1))
        chosen = torch.where(stop, pick, chosen)
        on = on & ~stop
        cur = torch.where(on, child, cur)
    path = torch.stack(path, 1)
    kept, past = (path >= 0).sum(1), lens - count
    # every accepted token's keys and values to its place; places that take none write the tree's first token to itself
    src = torch.where(path >= 0, past[:, None] + path, past[:, None])
    dst = torch.where(path >= 0, past[:, None] + torch.arange(most, device=DEV), past[:, None])
    src_page, dst_page = table.gather(1, src // PAGE), table.gather(1, dst // PAGE)
    pool[:, dst_page, :, :, dst % PAGE] = pool[:, src_page, :, :, src % PAGE]
    out = {"path": path, "counts": kept, "next": chosen, "new_lens": past + kept}
    return {**{k: v.int() for k, v in out.items()}, "pool": pool}


# ---- the same from the definitions, in 64 bits -------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    return {"rotate": _exact_rotate, "append": _exact_append, "tree": _exact_tree, "commit": _exact_commit}[case["kind"]](case, s)


def _exact_turn(case, positions, x):
    """Columns multiplied as complex numbers of modulus `scale`."""
    f, scale = _frequencies(case)
    heads, h = x.shape[1] // DIM, case["dim"] // 2
    y = x.double().reshape(-1, heads, DIM).clone()
    pos = positions.double()
    unit = torch.polar(torch.full((pos.numel(), h), scale, dtype=torch.float64, device=DEV),
                       pos[:, None] * torch.tensor(f, dtype=torch.float64, device=DEV))
    for i in range(h):
        a, b = (i, i + h) if case["layout"] == "halves" else (2 * i, 2 * i + 1)
        z = torch.complex(y[:, :, a].clone(), y[:, :, b].clone()) * unit[:, i:i + 1]
        y[:, :, a], y[:, :, b] = z.real, z.imag
    return y.flatten(1)


def _exact_rotate(case, s):
    return _exact_turn(case, s["positions"], s["x"])


def _exact_append(case, s):
    want, q_out = s["pool"].double(), s["q_out"].double()
    T = case["rows"]
    slots, pos = s["slots"][:T].long(), s["positions"][:T]
    for j, src in enumerate((_exact_turn(case, pos, s["k"][:T]), s["v"][:T].double())):
        for h in range(case["kv_heads"]):
            want[0, slots // PAGE, j, h, slots % PAGE] = src[:, h * DIM:(h + 1) * DIM]
    q_out[:T] = _exact_turn(case, pos, s["q"][:T])
    return {"pool": want, "q_out": q_out}


def _exact_tree(case, s):
    past, rows, _ = _lens(case)
    G, KH, P, pool = case["heads"] // case["kv_heads"], case["kv_heads"], case["prefix"], s["pool"][0]
    out = torch.zeros((sum(rows), case["heads"], DIM), dtype=torch.float64, device=DEV)
    words, t0 = s["masks"].cpu().numpy().astype("uint64").tolist(), 0
    for b, (c, n) in enumerate(zip(past, rows)):
        ids = torch.cat([s["prefix_pages"], s["table"][b, :_pages(c + n)]]).long()
        at = torch.cat([torch.arange(P, device=DEV), _pages(P) * PAGE + torch.arange(c + n, device=DEV)])
        hide = torch.zeros((n, P + c + n), dtype=torch.bool)
        for i in range(n):
            bits = sum(w << 64 * k for k, w in enumerate(words[t0 + i]))
            for j in range(n):
                hide[i, P + c + j] = not bits >> j & 1
        hide = hide.to(DEV)
        for h in range(KH):
            key, val = (pool[ids, j, h].reshape(-1, DIM)[at].double() for j in (0, 1))
            for k in range(h * G, h * G + G):
                x = (s["q"][t0:t0 + n, k * DIM:(k + 1) * DIM].double() @ key.T) * DIM ** -0.5
                out[t0:t0 + n, k] = torch.softmax(x.masked_fill_(hide, -math.inf), -1) @ val
        t0 += n
    return out.flatten(1)


def _exact_commit(case, s):
    past, rows, _ = _lens(case)
    tokens, parents, choices, table = (s[k].tolist() for k in ("tokens", "parents", "choices", "table"))
    want, most, t0 = s["pool"].double(), s["path"].shape[1], 0
    paths, counts, chosen = [], [], []
    for b, (c, n) in enumerate(zip(past, rows)):
        path = [0]
        while True:
            pick = choices[t0 + path[-1]]
            below = [j for j in range(path[-1] + 1, n) if parents[t0 + j] == path[-1] and tokens[t0 + j] == pick]
            if not below or len(path) == most:
                break
            path.append(below[0])
        old = [want[:, table[b][(c + p) // PAGE], :, :, (c + p) % PAGE].clone() for p in path]
        for i, x in enumerate(old):
            want[:, table[b][(c + i) // PAGE], :, :, (c + i) % PAGE] = x
        paths.append(path + [-1] * (most - len(path)))
        counts.append(len(path))
        chosen.append(pick)
        t0 += n
    return {"path": _i32(paths), "counts": _i32(counts), "next": _i32(chosen),
            "new_lens": _i32([c + k for c, k in zip(past, counts)]), "pool": want}


# ---- what a pass cannot do without ---------------------------------------------------------------
def work(case):
    size = {"bf16": 2, "f32": 4}
    if case["kind"] in ("rotate", "append"):
        T = case["rows"]
        turned, copied = (case["heads"], 0) if case["kind"] == "rotate" else (case["heads"] + case["kv_heads"], case["kv_heads"])
        n = T * DIM * (turned + copied)
        ints = T if case["kind"] == "rotate" else 2 * T + case["pad"]
        return {"bytes": n * (size[case["src"]] + size[case["dst"]]) + 4 * ints, "flops": 3 * T * turned * case["dim"]}
    past, rows, kept = _lens(case)
    if case["kind"] == "commit":
        moved = sum(k - 1 for k in kept) * case["layers"] * 2 * case["kv_heads"] * DIM * size[case["dtype"]]
        # three numbers a token are read, the paths and three numbers a sequence written
        return {"bytes": 2 * moved + 12 * sum(rows) + 4 * case["batch"] * (case["keep_hi"] + 1 + 5), "flops": 0}
    P, T = case["prefix"], sum(rows)
    keys = P + sum(c + n for c, n in zip(past, rows))
    # a row's tree tokens count as half the tree: its ancestors are fewer, but which is an input
    pairs = T * P + sum(n * c + n * (n + 1) // 2 for c, n in zip(past, rows))
    return {"bytes": size[case["dtype"]] * DIM * (2 * keys * case["kv_heads"] + 2 * T * case["heads"]) + 8 * T * _pages(max(rows)),
            "flops": 4 * DIM * case["heads"] * pairs}
