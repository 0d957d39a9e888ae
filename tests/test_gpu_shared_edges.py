"""Serving behind a shared prefix where it can go wrong: near-ties between large scores, values and
scores that are not finite, pages outside the pool, tables far wider than their sequences."""
import numpy as np
import pytest

from paper_2607_21042_amd import ftts, workload
from tests import helpers
from tests.test_gpu_paged import Batch, dev, kernel, reference64  # noqa: F401

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


# ---- the decode step's queries ----------------------------------------------------------------
ONE = workload.ModelShape(n_layer=1, d_model=256, n_head=4, d_head=64, d_ff=512, vocab=640)


def wide_model():
    """One layer whose queries are about 6 wide, whose out-projection is the identity and whose MLP adds
    nothing, on rows of 0.01: the hidden state is LayerNorm(the attention's output), near enough."""
    m, d = workload.master_weights(ONE, seed=11), ONE.d_model
    m["tok_emb"], m["pos_emb"] = m["tok_emb"] * 0.5, m["pos_emb"] * 0.5
    m["lnf_g"], m["lnf_b"] = np.ones_like(m["lnf_g"]), np.zeros_like(m["lnf_b"])
    w = m["layers"][0]
    w["w_qkv"] = w["w_qkv"].copy()
    w["w_qkv"][:d] *= 6.0 / (0.02 * np.sqrt(d))
    w["w_out"], w["b_out"] = np.eye(d, dtype=np.float32), np.zeros_like(w["b_out"])
    w["w_fc2"], w["b_fc2"] = np.zeros_like(w["w_fc2"]), np.zeros_like(w["b_fc2"])
    return workload.bf16_weights(m)


def queries(m, tokens, pos):
    x = m["tok_emb"][tokens].astype(np.float64) + m["pos_emb"][pos]
    w = m["layers"][0]
    n = (x - x.mean(1, keepdims=True)) / np.sqrt(x.var(1, keepdims=True) + 1e-5) * w["ln1_g"] + w["ln1_b"]
    return (n @ w["w_qkv"][:256].astype(np.float64).T + w["b_qkv"][:256]).reshape(len(tokens), 4, 64)


@pytest.mark.parametrize("B,P,own", [(1, 64, 3), (2, 192, 70), (3, 1984, 130), (8, 1280, 200), (24, 640, 66), (33, 320, 40)])
def test_decode_queries_keep_their_bits_behind_a_shared_prefix(B, P, own):
    """A decode step's fp32 query reaches the scores with 16 bits, as in the step without a prefix.  Each
    sequence and head has a token of its own whose score ties with the prefix's largest, among scores of
    some 100: a query of 8 bits moves such a pair against each other by 0.04 and more.

    The same pages serve as a shared prefix and as the first pages of every block table, so queries, keys
    and values of both calls are the same bits.  Bound: with S the largest sum_d |q_d k_d| / 8, the
    two-part query (2^-18 of itself) and the sum of 64 products in fp32 (64 u = 2^-18) shift a score by at
    most 2^-17 S; with scaling and exponential eps = 3 * 2^-18 S.  An output o moves by sum_j p_j ds_j
    (v_j - o), at most eps sum p |v - o| a side, sixteen-bit outputs by 2^-8 of themselves a side more, and
    LayerNorm, a projection and a scale, keeps errors relative to |o - mean| (5% for the rows it adds)."""
    m = wide_model()
    rng = np.random.default_rng(B)
    tokens, pos = rng.integers(0, ONE.vocab, B), np.full(B, 2)
    n_pre, n_own = P // 64, -(-(own + 1) // 64)
    n_pages = n_pre + B * n_own
    ids = rng.permutation(n_pages)
    pre, table = ids[:n_pre], ids[n_pre:].reshape(B, n_own)
    pool = np.zeros((1, n_pages, 2, 4, 64, 64), dtype=np.float32)
    pool[:, :, 0] = workload.bf16_round(rng.standard_normal((1, n_pages, 4, 64, 64)).astype(np.float32) * np.float32(6))
    pool[:, table, 0] = workload.bf16_round(pool[:, table, 0] * np.float32(0.5))   # (the prefix's largest stays the largest)
    pool[:, :, 1] = workload.bf16_round(rng.standard_normal((1, n_pages, 4, 64, 64)).astype(np.float32))
    q = queries(m, tokens, pos)
    move, out, S, near = np.zeros((B, 4, 64)), np.zeros((B, 4, 64)), 0.0, 0
    for b in range(B):
        for h in range(4):
            best = (pool[0, pre, 0, h].reshape(-1, 64) @ q[b, h]).max()
            t = int(rng.integers(0, own))
            k = rng.standard_normal(64) * 6
            k += (best - k @ q[b, h]) / (q[b, h] @ q[b, h]) * q[b, h]
            pool[0, table[b, t // 64], 0, h, t % 64] = workload.bf16_round(k.astype(np.float32))
            pg = np.concatenate([pre, table[b]])
            key, val = (pool[0, pg, j, h].reshape(-1, 64)[:P + own].astype(np.float64) for j in (0, 1))
            s = key @ q[b, h] / 8
            p = np.exp(s - s.max())
            p /= p.sum()
            near += np.sort(p)[-2] > 0.05
            out[b, h] = p @ val
            move[b, h] = p @ np.abs(val - out[b, h])
            S = max(S, (np.abs(key) @ np.abs(q[b, h])).max() / 8)
    assert near >= 2 * B
    dm = ftts.DeviceModel(m, ONE, ftts.BF16)
    cache = torch.from_numpy(pool).cuda().bfloat16()

    class View(ftts.KVCache):
        def __init__(self, pool):
            self.pool = pool
            self._view()

    hid = []
    for shared in (True, False):
        kv = View(cache.clone())
        bt = table if shared else np.concatenate([np.tile(pre, (B, 1)), table], 1)
        pt = ftts.PageTableView(dev(bt), dev(np.full(B, own + (0 if shared else P))))
        ws = torch.zeros(ftts.shared_workspace_bytes(dm.cfg, B, B, P, bt.shape[1]), dtype=torch.uint8, device="cuda")
        logits, ids_out = torch.empty((B, ONE.vocab), device="cuda"), dev(np.zeros(B))
        h = torch.empty((B, 256), device="cuda")
        kw = dict(hidden_out=h)
        greedy = ftts.Sampling(1.0, 1, 1.0)
        print(f"decode queries: B {B}, prefix {P}, {'shared' if shared else 'copied'}", flush=True)
        if shared:
            ftts.decode_step_shared(dm, ftts.SharedPrefix(dev(pre), P), dev(tokens), dev(pos), pt, kv, logits, ids_out, None,
                                    greedy, ws, **kw)
        else:
            ftts.decode_step(dm, dev(tokens), dev(pos), pt, kv, logits, ids_out, None, greedy, ws, **kw)
        torch.cuda.synchronize()
        hid.append((h.cpu().numpy().astype(np.float64), kv.pool))
    assert torch.equal(hid[0][1], hid[1][1])
    move, out = move.reshape(B, 256), out.reshape(B, 256)
    ratio = np.linalg.norm(move, axis=1) / np.linalg.norm(out - out.mean(1, keepdims=True), axis=1)
    bound = 1.05 * (2 * 3 * 2.0 ** -18 * S * ratio + 2 * 2.0 ** -8 * (B >= 5))  # (from 5 rows on the step's outputs are bf16)
    err = np.linalg.norm(hid[0][0] - hid[1][0], axis=1) / np.linalg.norm(hid[1][0], axis=1)
    print(f"error {err.max():.2e}, bound {bound.min():.2e}, S {S:.0f}", flush=True)
    assert (err <= bound).all(), (err / bound).max()


# ---- values and scores that are not finite ------------------------------------------------------
FORMS = [  # dtype, heads, prefix, own tokens before the rows, rows (None: one a sequence), the kernel
    ("bf16", 4, 4, 60, [3, 40, 200], None, "whole"), ("bf16", 5, 1, 60, [3, 40], None, "whole"),
    ("bf16", 4, 4, 4000, [70, 5], None, "cut"), ("bf16", 4, 4, 2500, [70, 5, 300, 1, 64, 90], None, "cut"),
    ("bf16", 10, 1, 3000, [70, 5], None, "cut"), ("f32", 4, 4, 70, [70, 5], None, "cut"),
    ("f32", 4, 4, 4000, [70, 5, 300, 1, 64, 90], None, "cut"), ("f32", 9, 1, 400, [70, 5], None, "cut"),
    ("bf16", 4, 4, 700, [20, 0], [40, 30], "cut"), ("f32", 4, 4, 700, [20, 0], [40, 30], "cut"),
    ("bf16", 8, 8, 70, [10] * 12, [90] * 12, "tile"), ("bf16", 20, 20, 333, [0] * 40, [40] * 40, "packed"),
    ("bf16", 12, 4, 2500, [10, 0, 300], [90, 130, 90], "packed in 8"), ("bf16", 20, 4, 2000, [0, 64, 700], [90, 128, 129], "tile in 4")]


def form(dtype, H, KH, prefix, past, rows, takes, **kw):
    lens = past if rows is None else [p + n for p, n in zip(past, rows)]
    b = Batch(dtype, H, KH, prefix, lens, rows, layers=1, **kw).gpu()
    assert kernel(b) == takes
    print(f"{takes}: {dtype} {H}/{KH} heads, prefix {prefix}, {len(lens)} sequences", flush=True)
    return b


def place(b, seq, tok):
    """(page, slot) of token `tok` of sequence seq, or of the prefix (seq None)."""
    return (b.pre if seq is None else b.table[seq])[tok // 64], tok % 64


def seen(b, seq, tok):
    """Rows that see the token: a slice of rows of the batch for a sequence's own, all for the prefix's."""
    if seq is None:
        return slice(0, b.T)
    if b.rows is None:
        return slice(seq, seq + 1)
    return slice(int(b.cu[seq]) + max(tok - (b.lens[seq] - b.rows[seq]), 0), int(b.cu[seq + 1]))


@pytest.mark.parametrize("dtype,H,KH,prefix,past,rows,takes", FORMS)
def test_an_infinite_value_is_infinite_where_it_is_seen(dtype, H, KH, prefix, past, rows, takes):
    """p * inf = inf for a weight above 0, in its dim alone: one in the prefix, one of a sequence's own tokens."""
    b = form(dtype, H, KH, prefix, past, rows, takes)
    b.call()
    torch.cuda.synchronize()
    want = b.out.view(b.T, H, 64).clone()
    own = 1 if rows is None else past[0] + rows[0] // 2
    for seq, tok, dim, what in ((None, min(prefix - 1, 37), 5, float("inf")), (None, prefix - 1, 40, float("-inf")),
                                (0, own, 63, float("-inf")), (0, own, 17, float("inf"))):
        pg, slot = place(b, seq, tok)
        b.kv.pool[0, pg, 1, :, slot, dim] = what
        want[seen(b, seq, tok), :, dim] = what
    b.call()
    torch.cuda.synchronize()
    assert torch.equal(b.out.view(b.T, H, 64), want)


@pytest.mark.parametrize("dtype,H,KH,prefix,past,rows,takes", FORMS)
def test_rows_whose_every_score_is_minus_infinity(dtype, H, KH, prefix, past, rows, takes):
    """Such a row has no softmax: NaN, where a row that sees no token is 0.  Tokens with a score of -inf next
    to others weigh nothing, wherever they are."""
    b = form(dtype, H, KH, prefix, past, rows, takes)
    b.qd.abs_().add_(0.25)
    clean = b.kv.pool.clone()
    pages = torch.from_numpy(b.pre).cuda()
    own = torch.from_numpy(b.table[b.table >= 0]).cuda()
    # all of them
    b.kv.pool[:, :, 0] = -float("inf")
    b.call()
    torch.cuda.synchronize()
    assert torch.isnan(b.out.float()).all()
    # the prefix's: what the call without a prefix gives; the first own page's: what is left is finite
    b.kv.pool.copy_(clean)
    b.kv.pool[:, pages, 0] = -float("inf")
    b.call()
    torch.cuda.synchronize()
    got = b.out.clone()
    alone, none = torch.empty_like(b.out), torch.full_like(b.ws, 0xFF)
    ftts.shared_attention(b.qd[:, :H * 64], b.kv, 0, b.pt, None, alone, none, row_offsets=b.cud)
    torch.cuda.synchronize()
    assert torch.isfinite(got.float()).all()
    err = (got.float() - alone.float()).norm() / alone.float().norm()
    assert err <= (2e-5 if dtype == "f32" else 2.0 ** -7), err    # (each is within half of that of the exact result)
    b.kv.pool.copy_(clean)
    b.kv.pool[:, own, 0] = -float("inf")
    b.call()
    torch.cuda.synchronize()
    got = b.out.clone()
    few = ftts.PageTableView(torch.full_like(b.pt.block_table, -1), b.pt.seq_lens)
    ftts.shared_attention(b.qd[:, :H * 64], b.kv, 0, few, b.prefix, alone, none, row_offsets=b.cud)
    torch.cuda.synchronize()
    err = (got.float() - alone.float()).norm() / alone.float().norm()
    assert torch.isfinite(got.float()).all() and err <= (2e-5 if dtype == "f32" else 2.0 ** -7), err
    # a row that sees no token, next to those: no page of sequence 0 is in the pool, and the prefix is none
    b.kv.pool[:, :, 0] = -float("inf")
    b.pt.block_table[0] = -1
    ftts.shared_attention(b.qd[:, :H * 64], b.kv, 0, b.pt, None, alone, none, row_offsets=b.cud)
    torch.cuda.synchronize()
    first = slice(0, 1 if rows is None else rows[0])
    assert (alone[first] == 0).all() and torch.isnan(alone[first.stop:].float()).all()


@pytest.mark.parametrize("dtype,H,KH,prefix,past,rows,takes", [f for f in FORMS if f[5]])
def test_a_value_that_is_not_finite_counts_at_a_weight_of_zero(dtype, H, KH, prefix, past, rows, takes):
    """0 * NaN = NaN, in a tile that some rows see in part as in the others; rows before the token keep their bits."""
    b = form(dtype, H, KH, prefix, past, rows, takes)
    b.qd.abs_().add_(0.25)
    pg, slot = place(b, 0, past[0] + rows[0] // 2)
    b.kv.pool[0, pg, 0, :, slot] = -300.0        # a score below -600: its weight is below 2^-800
    b.call()
    torch.cuda.synchronize()
    want = b.out.clone()
    assert torch.isfinite(want.float()).all()
    b.kv.pool[0, pg, 1, :, slot] = float("nan")
    want[seen(b, 0, past[0] + rows[0] // 2)] = float("nan")
    b.call()
    torch.cuda.synchronize()
    assert torch.equal(b.out.float().nan_to_num(123.0), want.float().nan_to_num(123.0))


# ---- pages outside the pool, wide tables ----------------------------------------------------------
@pytest.mark.parametrize("H,KH,prefix,past,rows,takes", [
    (12, 4, 2500, [10, 0, 300], [90, 130, 90], "packed in 8"), (20, 4, 2000, [0, 64, 3, 700], [90, 0, 128, 129], "tile in 4"),
    (20, 20, 0, [2900], [300], "tile in 4")])
def test_parts_with_pages_outside_the_pool(H, KH, prefix, past, rows, takes):
    """A page of the prefix, an own page and a sequence of fewer tokens than rows, where a tile's chain is cut."""
    b = Batch("bf16", H, KH, prefix, [p + n for p, n in zip(past, rows)], rows, extra_rows=2, layers=1)
    if prefix:
        b.pre = b.pre.copy()
        b.pre[len(b.pre) // 2], b.pre[0] = b.pool.shape[1], -1
    b.table[-1, 2], b.table[0, 0] = 2 ** 31 - 1, -7
    b.lens[0] = rows[0] - 40 if len(rows) > 1 else b.lens[0]
    b.gpu()
    assert kernel(b) == takes
    print(f"{takes}: pages outside the pool, {H}/{KH} heads, prefix {prefix}, rows {rows}", flush=True)
    b.call()
    b.check()


@pytest.mark.parametrize("dtype,H,KH,prefix,lens,rows", [
    ("bf16", 20, 20, 300, [700, 0, 1, 64, 65, 513, 129, 300] * 4, None), ("f32", 20, 20, 130, [700, 0, 1, 513, 129, 300], None),
    ("bf16", 20, 4, 0, [1200, 33, 7] * 21, None), ("bf16", 6, 3, 65, [90, 1, 300], [3, 1, 40]),
    ("f32", 4, 2, 65, [90, 1, 300], [3, 1, 40]), ("bf16", 20, 20, 700, [200, 260], [120, 200])])
def test_tables_far_wider_than_their_sequences(dtype, H, KH, prefix, lens, rows):
    """512 pages a sequence, as a server's table may have: runs of own pages grow with the table."""
    b = Batch(dtype, H, KH, prefix, lens, rows, layers=1, width=512).gpu()
    print(f"wide table: {dtype} {H}/{KH} heads, prefix {prefix}, {len(lens)} sequences: {kernel(b)}", flush=True)
    b.call()
    b.check()
