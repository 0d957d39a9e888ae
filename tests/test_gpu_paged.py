"""Block tables, KV append and shared-prefix attention against the numpy oracle (float64).

Tables and appended rows are compared bit for bit.  Attention: with u = 2^-24, a score is a sum of
64 products, scaled and shifted, so it is off by at most about 82 u times the largest
sum_d |q_d k_d| / 8 of its row (the hardware exponential adds a few u), and a weighted mean over n
tokens by at most (2 eps_p + 2 (n + 16) u) sum p |v| / sum p.  In bf16 the weights are rounded
once (numerator and sum: 2^-8 of sum p |v| / sum p each) and the output once (2^-8 of itself).
Those are worst cases; norms over a whole output see independent roundings: two of 2^-8 / sqrt(3)
times at most one give below 2^-8 in bf16.
"""
import numpy as np
import pytest

from oracle import paged
from paper_2607_21042_amd import ftts, workload

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
U = 2.0 ** -24


def dev(a, dtype=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda().to(dtype)


# ---- tables ---------------------------------------------------------------------------------
def run_tables(cached, added, free, n_pages, old, max_rows, with_lens=True):
    B = len(added)
    t = dict(table=dev(old), cu=dev(np.full(B + 1, -7)), lens=dev(np.full(B, -7)), slots=dev(np.full(max_rows, -7)),
             counts=dev(np.full(2, -7)))
    ftts.build_tables(dev(added), dev(np.asarray(free, dtype=np.int64)), n_pages, t["table"], t["cu"], t["slots"],
                      t["counts"], cached=None if cached is None else dev(cached), seq_lens=t["lens"] if with_lens else None)
    torch.cuda.synchronize()
    return {k: v.cpu().numpy() for k, v in t.items()}


def check_tables(cached, added, free, n_pages, old, max_rows):
    got = run_tables(cached, added, free, n_pages, old, max_rows)
    want = paged.build_tables(np.zeros(len(added)) if cached is None else cached, added, free, n_pages, old, max_rows)
    for k, w in zip(("table", "cu", "lens", "slots", "counts"), want):
        assert np.array_equal(got[k], w), k


@pytest.mark.parametrize("B,width,hi_c,hi_a,spare", [
    (1, 1, 0, 64, 0), (1, 512, 20000, 9000, 3), (3, 4, 100, 100, 0), (63, 9, 300, 200, -5), (64, 9, 300, 1, 0),
    (65, 20, 600, 600, 7), (200, 30, 1900, 0, 0), (1023, 12, 700, 40, -300), (1024, 24, 0, 1500, 1)])
def test_tables_ragged(B, width, hi_c, hi_a, spare):
    rng = np.random.default_rng(B * 7 + width)
    cached, added = rng.integers(0, hi_c + 1, B), rng.integers(0, hi_a + 1, B)
    total = int((-(-(cached + added) // 64) - -(-cached // 64)).sum())
    n_pages = 5000 + B * width
    free = rng.permutation(n_pages)[:max(0, total + spare)]
    old = rng.integers(0, n_pages, (B, width))
    print(f"tables: B {B}, width {width}", flush=True)
    check_tables(cached, added, free, n_pages, old, int(added.sum()) + 17)
    check_tables(None, added, free, n_pages, old, max(0, int(added.sum()) - 5))


def test_tables_refusals_on_the_device():
    """Negative and too long requests, lengths at the ends of int32, pages outside the pool, no free pages."""
    old = np.arange(24).reshape(8, 3)
    big = 2 ** 31 - 1
    for cached, added in (([0, -1, 5, 64, 192, 193, big, -big - 1], [64, 3, -2, 65, 0, 0, 1, 7]),
                          ([0, 0, 0, 1, 2, 3, 0, 0], [big, big, big, big, 64, big, 1, 1]),
                          ([0] * 8, [0] * 8)):
        for free in ([30, 31, 99, 32, 33, 34, 35], [30], []):
            check_tables(np.array(cached), np.array(added), free, 60, old, 150)
    got = run_tables(None, np.array([5, 70]), [3, 4, 5], 60, np.full((2, 3), 9), 0, with_lens=False)
    assert got["cu"].tolist() == [0, 5, 75] and got["table"].tolist() == [[3, -1, -1], [4, 5, -1]]
    assert (got["lens"] == -7).all()


# ---- append ---------------------------------------------------------------------------------
@pytest.mark.parametrize("src,dst", [("bf16", "bf16"), ("f32", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("T,H,packed", [(1, 1, False), (3, 4, True), (64, 20, True), (130, 12, False), (257, 5, True)])
def test_append(src, dst, T, H, packed):
    rng = np.random.default_rng(T * H)
    st, dt = (torch.bfloat16 if x == "bf16" else torch.float32 for x in (src, dst))
    n_pages = T // 64 + 3
    width = (3 if packed else 2) * H * 64
    rows = rng.standard_normal((T, width)).astype(np.float32)
    if src == "bf16":
        rows = workload.bf16_round(rows)
    slots = rng.permutation(n_pages * 64)[:T]
    slots[::5] = rng.choice([-1, -70, n_pages * 64, 2 ** 31 - 1], len(slots[::5])) if T > 1 else slots[::5]
    old = workload.bf16_round(rng.standard_normal((2, n_pages, 2, H, 64, 64)).astype(np.float32))
    x, pool = torch.from_numpy(rows).cuda().to(st), torch.from_numpy(old).cuda().to(dt)
    k, v = x[:, -2 * H * 64:-H * 64], x[:, -H * 64:]
    print(f"append: {src} -> {dst}, {T} rows, {H} heads", flush=True)
    ftts.append_kv(k, v, dev(slots), ftts.KVCache.over(pool), 1)
    torch.cuda.synchronize()
    new = workload.bf16_round(rows) if dst == "bf16" else rows
    want = paged.append(old, 1, new[:, -2 * H * 64:-H * 64], new[:, -H * 64:], slots)
    assert np.array_equal(pool.float().cpu().numpy(), want)


def test_append_keeps_infinities_and_nan():
    pool = torch.zeros((1, 1, 2, 1, 64, 64), device="cuda", dtype=torch.bfloat16)
    k = torch.full((2, 64), float("nan"), device="cuda")
    v = torch.full((2, 64), -3.4e38, device="cuda")     # beyond bf16: rounds to -inf
    v[1] = float("inf")
    ftts.append_kv(k, v, dev([5, 6]), ftts.KVCache.over(pool), 0)
    torch.cuda.synchronize()
    assert torch.isnan(pool[0, 0, 0, 0, 5:7]).all() and (pool[0, 0, 1, 0, 6] == float("inf")).all()
    assert (pool[0, 0, 1, 0, 5] == v[0].bfloat16()).all() and (pool[0, 0, :, 0, 7:] == 0).all()


# ---- attention ------------------------------------------------------------------------------
class Batch:
    """Random queries, pool (NaN wherever no token is), tables; rows: None for one a sequence."""

    def __init__(self, dtype, H, KH, prefix, lens, rows=None, extra_rows=0, packed=False, seed=0, spread=0.7, layers=2,
                 width=None):
        rng = np.random.default_rng([seed, prefix, H])
        self.f32, self.H, self.KH, self.P, self.lens = dtype == "f32", H, KH, prefix, list(lens)
        self.t = torch.float32 if self.f32 else torch.bfloat16
        B = len(lens)
        need = [-(-max(n, 0) // 64) for n in lens]
        n_pre = -(-prefix // 64)
        self.width = width or max(max(need), 1)
        n_pages = n_pre + sum(need) + 2
        ids = rng.permutation(n_pages)
        self.pre = ids[:n_pre]
        self.table = np.full((B, self.width), -1, dtype=np.int64)
        self.layer = layers - 1
        self.pool = np.full((layers, n_pages, 2, KH, 64, 64), np.nan, dtype=np.float32)
        at = n_pre
        tokens = [(self.pre[t // 64], t % 64) for t in range(prefix)]
        for b, n in enumerate(need):
            k = min(n, self.width)
            self.table[b, :k] = ids[at:at + k]
            at += n
            tokens += [(self.table[b, t // 64], t % 64) for t in range(min(max(lens[b], 0), 64 * self.width))]
        values = rng.standard_normal((len(tokens), 2, KH, 64)).astype(np.float32) * np.float32(spread)
        if tokens:
            pg, sl = np.array(tokens).T
            self.pool[self.layer, pg, :, :, sl] = values if self.f32 else workload.bf16_round(values)
        self.rows = rows
        self.cu = None if rows is None else np.concatenate([[0], np.cumsum(rows)])
        self.T = (B if rows is None else sum(rows)) + extra_rows
        q = rng.standard_normal((self.T, (3 if packed else 1) * H * 64)).astype(np.float32) * np.float32(spread)
        self.q = q if self.f32 else workload.bf16_round(q)

    def gpu(self):
        self.qd = torch.from_numpy(self.q).cuda().to(self.t)
        self.kv = ftts.KVCache.over(torch.from_numpy(self.pool).cuda().to(self.t))
        self.pt = ftts.PageTableView(dev(self.table), dev(self.lens))
        self.prefix = ftts.SharedPrefix(dev(self.pre), self.P) if self.P else None
        self.cud = None if self.cu is None else dev(self.cu)
        self.out = torch.full((self.T, self.H * 64), -7.0, device="cuda", dtype=self.t)
        self.ws = torch.full((ftts.shared_attention_workspace_bytes(self.H, self.KH, self.kv.dtype, len(self.lens), self.T,
                                                                    self.P, self.width),), 0xFF, dtype=torch.uint8, device="cuda")
        return self

    def call(self, **kw):
        ftts.shared_attention(self.qd[:, :self.H * 64], self.kv, self.layer, self.pt, self.prefix, self.out, self.ws,
                              row_offsets=self.cud, **kw)

    def check(self):
        ref, size, dots, n = paged.shared_attention(self.q[:, :self.H * 64].reshape(self.T, self.H, 64), self.pool[self.layer],
                                                    self.pre, self.P, self.table, self.lens, self.cu, weights=True)
        got = self.out.float().cpu().numpy().reshape(ref.shape)
        none = np.isnan(ref)
        assert (got[none] == -7.0).all(), "a row of no sequence was written"
        eps = 82 * U * dots[:, :, None] + 8 * U
        bound = (2 * eps + 2 * U * (n[:, None, None] + 16)) * size
        if not self.f32:
            bound = bound + 2.0 ** -8 * (2 * size + np.abs(ref))
        err = np.abs(got - ref)[~none]
        over = err - bound[~none]
        assert np.isfinite(err).all() and (over <= 0).all(), (err.max(), over.max())
        rel = np.linalg.norm(err) / max(np.linalg.norm(ref[~none]), 1e-30)
        assert rel <= (1e-5 if self.f32 else 2.0 ** -8), rel
        return rel


def kernel(b):
    """Which of the launcher's kernels a call takes: "whole" (one row a sequence, one launch), "tile" (128 rows of a
    sequence share pages, one launch), "packed" (128 rows of all), either of them " in" parts that are joined, or "cut"
    (tiles of 32 or fewer, along the tokens, joined); fp32 is always cut."""
    if b.f32:
        return "cut"
    B, g, pages, own = len(b.lens), b.H // b.KH, -(-b.P // 64), b.width
    if b.cu is None:
        tiles = B * -(-g // 32)
        whole = 3.5 + 0.32 * (pages + own) * max(1.0, tiles * b.KH / 240)
        fits = pages + own <= 256 and whole <= 8.5 + 1.3e-3 * b.KH * (pages * -(-B * g // 32) + tiles * min(own, 16))
        return "whole" if fits else "cut"
    pairs, tiles = b.T * g, -(-b.T * g // 128)
    least, name = 9.0 + 1.65e-3 * b.KH * (-(-pairs // 32) * pages + 0.8 * (pairs / 32 + B) * own) + 0.53e-3 * b.T * b.H, "cut"
    for pack in (False, True):
        units = b.KH * (tiles if pack else pairs / 128 + 0.5 * B) / 256
        chain = pages + 1.1 * own * (1 + (B - 1) / tiles if pack else 1)
        for parts in (1, 2, 4, 8, 16):
            if parts > 1 and (4 * parts > pages + own or (tiles if pack else pairs // 128 + B) * b.KH * parts > 2048):
                break
            rate, u = 1.1 if pack else 1.0, units * parts
            t = 5.5 + 0.8 * rate * chain * max(1.0, u)
            if parts > 1:
                t = 13 + 0.7 * rate * (chain / parts + 0.5) * max(1.0, 0.5 * (u + np.ceil(u))) + 0.03e-3 * parts * b.T * b.H
            if t < least or (t == least and not pack):
                least, name = t, ("packed" if pack else "tile") + (f" in {parts}" if parts > 1 else "")
    return name


def test_the_cases_take_every_kernel():
    one = {kernel(Batch("bf16", H, KH, P, EDGE)) for H, KH in HEADS for P in (0, 1, 63, 64, 65, 130, 700)}
    few = {kernel(Batch("bf16", 4, 4, P, [1, 2, 33, 7], [1, 2, 33, 7])) for P in (0, 65, 400)}
    wide = {kernel(Batch("bf16", H, KH, P, r, r)) for H, KH, P, r in ((8, 8, 150, [120] * 12 + [1, 129]), (20, 20, 33, [40] * 20))}
    assert one == {"whole", "cut"} and few == {"tile", "cut"} and wide == {"tile"}


EDGE = [0, 1, 2, 63, 64, 65, 127, 128, 129, 200, 256, 257, 321, 500, 513, 700]
HEADS = [(4, 4), (5, 1), (6, 3)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,KH", HEADS)
@pytest.mark.parametrize("prefix", [0, 1, 63, 64, 65, 130, 700])
def test_single_token(dtype, H, KH, prefix):
    b = Batch(dtype, H, KH, prefix, EDGE, packed=prefix % 2 == 1).gpu()
    print(f"single token: {dtype} {H}/{KH} heads, prefix {prefix}", flush=True)
    b.call()
    b.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,KH,B,prefix,longest", [(5, 1, 6, 5000, 1200), (4, 2, 3, 4333, 300), (1, 1, 2, 8190, 1300),
                                                   (1, 1, 1, 12300, 64), (2, 1, 40, 2500, 700), (3, 3, 1, 4700, 520)])
def test_many_partial_results(dtype, H, KH, B, prefix, longest):
    """Long prefixes and wide tables: from 17 to over 64 runs of pages a row, in numbers that four do not divide."""
    lens = np.random.default_rng(prefix).integers(0, longest + 1, B)
    lens[0] = longest
    b = Batch(dtype, H, KH, prefix, lens.tolist()).gpu()
    print(f"many partials: {dtype} {H}/{KH} heads, B {B}, prefix {prefix}", flush=True)
    b.call()
    b.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,prefix,lens", [(1, 0, [1]), (1, 1, [0]), (1, 300, [40]), (2, 5, [3, 900]), (33, 90, None),
                                           (64, 260, None)])
def test_single_token_batches(dtype, B, prefix, lens):
    rng = np.random.default_rng(B)
    b = Batch(dtype, 3, 3, prefix, lens or rng.integers(-2, 150, B).tolist()).gpu()
    print(f"single token batch: {dtype} B {B}, prefix {prefix}", flush=True)
    b.call()
    b.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,KH,B,prefix", [(4, 1, 3, 70), (8, 1, 1, 900), (16, 2, 3, 900), (9, 1, 2, 900), (17, 1, 5, 40),
                                           (33, 1, 3, 0), (40, 1, 2, 1500)])
def test_many_query_heads_a_key_head(dtype, H, KH, B, prefix):
    """Rows that fill their tiles of 4 and 32, pass them by one, and need several."""
    b = Batch(dtype, H, KH, prefix, [70, 300, 1, 0, 513][:B]).gpu()
    print(f"query heads: {dtype} {H}/{KH}, B {B}, prefix {prefix}: {kernel(b)}", flush=True)
    b.call()
    b.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,KH", HEADS)
@pytest.mark.parametrize("prefix", [0, 65, 400])
@pytest.mark.parametrize("past,rows", [
    ([0, 0, 0, 0], [1, 2, 33, 7]), ([0, 5, 63, 64], [64, 65, 31, 1]), ([130, 0, 1, 200, 9], [3, 0, 0, 8, 1]), ([0], [150])])
def test_prompt_rows(dtype, H, KH, prefix, past, rows):
    lens = [p + n for p, n in zip(past, rows)]
    b = Batch(dtype, H, KH, prefix, lens, rows, extra_rows=3, packed=prefix == 65).gpu()
    print(f"prompt rows: {dtype} {H}/{KH} heads, prefix {prefix}, rows {rows}", flush=True)
    b.call()
    b.check()


@pytest.mark.parametrize("dtype,H,KH,prefix,rows", [
    ("bf16", 8, 8, 150, [120] * 12 + [1, 129]), ("bf16", 10, 2, 65, [200, 5, 130]), ("bf16", 20, 20, 33, [40] * 20),
    ("f32", 4, 4, 130, [70, 33])])
def test_prompt_rows_of_wider_batches(dtype, H, KH, prefix, rows):
    b = Batch(dtype, H, KH, prefix, [n + 10 * (i % 3) for i, n in enumerate(rows)], rows).gpu()
    print(f"wide prompt: {dtype} {H}/{KH} heads, {len(rows)} sequences", flush=True)
    b.call()
    b.check()


def packed_batch(H, KH, prefix, B, longest, seed):
    """Short prompts in tiles of 128 rows that go over sequences' ends: sequences without rows, of one row, with cached
    tokens, inactive, with fewer tokens than rows, rows before the first sequence and behind the last."""
    rng = np.random.default_rng(seed)
    rows = rng.integers(1, longest + 1, B).tolist()
    rows[0], rows[5], rows[6], rows[7], rows[B - 1] = 1, 0, 0, 130, 2
    lens = [n + (int(rng.integers(0, 100)) if i % 6 == 1 else 0) for i, n in enumerate(rows)]
    b = Batch("bf16", H, KH, prefix, lens, rows, extra_rows=7, seed=seed, layers=1)
    b.lens[3], b.lens[9], b.lens[10] = -1, rows[9] - 1, 0
    b.cu = b.cu + 3
    return b


@pytest.mark.parametrize("H,KH,prefix,B,longest", [
    (20, 20, 333, 40, 80), (20, 20, 64, 40, 70), (24, 8, 500, 64, 50), (18, 6, 1000, 64, 60), (32, 16, 1, 64, 70)])
def test_prompts_that_share_row_tiles(H, KH, prefix, B, longest):
    b = packed_batch(H, KH, prefix, B, longest, 3).gpu()
    takes = kernel(b)
    print(f"packed prompts: {H}/{KH} heads, prefix {prefix}, {B} sequences: {takes}", flush=True)
    assert takes == ("packed" if prefix > 64 else "tile")
    b.call()
    torch.cuda.synchronize()
    for seq in range(B):
        if b.rows[seq] and b.lens[seq] >= 0:
            ref, got = reference64(b, seq, list(range(b.rows[seq])))
            assert (got - ref).norm() <= 2.0 ** -8 * ref.norm() and (got - ref).abs().max() <= 2.0 ** -7 * ref.abs().max(), seq
    assert (b.out[b.cu[3]:b.cu[4]] == 0).all()
    assert (b.out[:3] == -7).all() and (b.out[-4:] == -7).all()


def test_prompts_that_share_row_tiles_over_many_pages():
    """Chains whose 64th page is one of the prefix, or in the middle of the sequences' own ones."""
    for prefix, B, takes in ((64 * 61 + 5, 64, "packed"), (64 * 70, 64, "packed"), (64 * 61 + 5, 40, "packed in 4"), (64 * 70, 40, "packed in 4")):
        b = packed_batch(20, 20, prefix, B, 60, 8).gpu()
        assert kernel(b) == takes
        print(f"{takes}: prompts behind {prefix}", flush=True)
        b.call()
        torch.cuda.synchronize()
        for seq in (0, 1, 7, 20, B - 1):
            ref, got = reference64(b, seq, sorted({0, b.rows[seq] // 2, b.rows[seq] - 1}))
            assert (got - ref).norm() <= 2.0 ** -8 * ref.norm(), seq
        assert (b.out[b.cu[3]:b.cu[4]] == 0).all()
        assert (b.out[:3] == -7).all() and (b.out[-4:] == -7).all()


@pytest.mark.parametrize("H,KH,prefix,past,rows,takes", [
    (12, 4, 2500, [10, 0, 300], [90, 130, 90], "packed in 8"), (20, 4, 2000, [0, 64, 3, 700], [90, 0, 128, 129], "tile in 4"),
    (20, 20, 0, [2900], [300], "tile in 4")])
def test_prompts_whose_pages_are_cut_into_parts(H, KH, prefix, past, rows, takes):
    """Parts that end inside the prefix and inside the own pages, an inactive sequence, a page outside the pool."""
    b = Batch("bf16", H, KH, prefix, [p + n for p, n in zip(past, rows)], rows, extra_rows=2, packed=True, layers=1).gpu()
    assert kernel(b) == takes
    print(f"{takes}: {H}/{KH} heads, prefix {prefix}, rows {rows}", flush=True)
    b.call()
    torch.cuda.synchronize()
    for seq in range(len(rows)):
        if rows[seq]:
            ref, got = reference64(b, seq, list(range(rows[seq])))
            assert (got - ref).norm() <= 2.0 ** -8 * ref.norm() and (got - ref).abs().max() <= 2.0 ** -7 * ref.abs().max(), seq
    assert (b.out[-2:] == -7).all()
    again = b.out.clone()
    b.ws.fill_(0xFF)
    b.call()
    assert torch.equal(b.out, again)
    b.lens[-1] = -1
    b.pt.seq_lens.copy_(dev(b.lens))
    b.call()
    torch.cuda.synchronize()
    assert (b.out[b.cu[-2]:b.cu[-1]] == 0).all()
    # (a shorter chain has other parts, which round otherwise: both are within 2^-8 of the exact result, as above)
    x, y = b.out[:b.cu[-2]].float(), again[:b.cu[-2]].float()
    assert (x - y).norm() <= 2.0 ** -7 * y.norm()


@pytest.mark.parametrize("prefix,takes", [(333, "packed"), (64 * 61 + 5, "packed in 4")])
def test_values_that_are_not_finite_stay_with_their_sequence(prefix, takes):
    """A sequence's own page of NaN and infinities changes no row of the others in its row tile, nor of an inactive
    sequence a prefix's."""
    b = packed_batch(20, 20, prefix, 40, 80 if prefix < 1000 else 60, 5).gpu()
    assert kernel(b) == takes
    b.call()
    clean = b.out.clone()
    r = slice(int(b.cu[4]), int(b.cu[5]))
    for what in (float("nan"), float("inf")):
        pool = b.pool.copy()
        pool[0, b.table[4, 0], 1, :, 0] = what
        b.kv.pool.copy_(torch.from_numpy(pool))
        b.call()
        torch.cuda.synchronize()
        assert torch.equal(b.out[:r.start], clean[:r.start]) and torch.equal(b.out[r.stop:], clean[r.stop:])
        assert not torch.isfinite(b.out[r].float()).any()
    pool = b.pool.copy()
    pool[0, b.pre[1], :, :, 7] = np.nan
    b.kv.pool.copy_(torch.from_numpy(pool))
    b.call()
    torch.cuda.synchronize()
    assert (b.out[b.cu[3]:b.cu[4]] == 0).all() and torch.isnan(b.out[r].float()).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_scores(dtype):
    """Scores far from zero and from each other (spread 6: |q . k| / 8 up to about 150) stay exact."""
    b = Batch(dtype, 4, 4, 200, [5, 64, 130], spread=6.0).gpu()
    b.call()
    b.check()
    b = Batch(dtype, 4, 2, 200, [40, 150], [40, 70], spread=6.0).gpu()
    b.call()
    b.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [None, [1, 2, 3, 40, 1]])
def test_rows_that_see_nothing(dtype, rows):
    """No prefix; lengths of 0 and below the rows (those before the first token see nothing), an inactive
    sequence, pages outside the pool, a length past the table."""
    b = Batch(dtype, 4, 2, 0, [0, 1, 2, 100, 150], rows, width=2).gpu()
    b.lens = [0, 1, -1, 100, 150]
    b.table[3, 1], b.table[1, 0] = 10 ** 6, -5
    b.gpu()
    print(f"empty rows: {dtype} {rows}", flush=True)
    b.call()
    b.check()
    if rows is not None:
        assert (b.out[:6] == 0).all()
    # behind a prefix with a page outside the pool
    p = Batch(dtype, 4, 2, 150, [0, 1, 2, 100, 150], rows, width=2)
    p.pre = p.pre.copy()
    p.pre[1] = 2 ** 31 - 1
    p.lens = [0, 1, -1, 100, 150]
    p.gpu().call()
    p.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,KH,B,prefix", [(4, 4, 2, 70), (8, 8, 12, 70), (6, 1, 2, 70), (4, 4, 1, 900), (6, 3, 2, 600),
                                           (12, 4, 3, 2500)])
def test_values_that_are_not_finite_reach_only_rows_that_see_them(dtype, H, KH, B, prefix):
    rows = [90] * B
    b = Batch(dtype, H, KH, prefix, [100] * B, rows).gpu()
    assert kernel(b) == ("cut" if dtype == "f32" or 70 < prefix < 1000 else "tile in 8" if prefix > 1000 else "tile")
    b.call()
    clean = b.out.clone()
    for tok, what in ((100 - 90 + 45, float("nan")), (99, float("inf")), (10 + 63, float("-inf")), (10 + 1, float("inf"))):
        pool = b.pool.copy()
        for j in (0, 1):  # key and value of one token of sequence 0
            pool[b.layer, b.table[0, tok // 64], j, :, tok % 64] = what if j else np.nan
        b.kv.pool.copy_(torch.from_numpy(pool))
        b.call()
        torch.cuda.synchronize()
        first = tok - 10                        # the first row that sees the token
        assert torch.equal(b.out[:first], clean[:first]) and torch.equal(b.out[90:], clean[90:]), tok
        assert torch.isnan(b.out[first:90].float()).all(), tok
        # an infinite value behind a finite key: infinite or NaN where it is seen, nothing elsewhere
        pool[b.layer, b.table[0, tok // 64], 0, :, tok % 64] = 0.25
        b.kv.pool.copy_(torch.from_numpy(pool))
        b.call()
        torch.cuda.synchronize()
        assert torch.equal(b.out[:first], clean[:first]) and torch.equal(b.out[90:], clean[90:]), tok
        assert not torch.isfinite(b.out[first:90].float()).any(), tok


def reference64(b, seq, rows):
    """Rows `rows` of sequence `seq` (indices within it) in float64 on the GPU, all heads."""
    n = 1 if b.rows is None else b.rows[seq]
    at = [(b.pre[t // 64], t % 64) for t in range(b.P)] + [(b.table[seq, t // 64], t % 64) for t in range(b.lens[seq])]
    pg, sl = (dev(x, torch.int64) for x in np.array(at).T)
    k, v = (b.kv.pool[b.layer][pg, j, :, sl].double().repeat_interleave(b.H // b.KH, 1) for j in (0, 1))
    first = seq if b.cu is None else int(b.cu[seq])
    q = b.qd[first + torch.tensor(rows, device="cuda"), :b.H * 64].double().view(len(rows), b.H, 64)
    out = torch.empty_like(q)
    for h in range(b.H):
        s = q[:, h] @ k[:, h].T / 8
        seen = (b.P + b.lens[seq] - n + torch.tensor(rows, device="cuda") + 1).clamp(min=b.P)
        s = s.masked_fill(torch.arange(len(pg), device="cuda")[None] >= seen[:, None], -float("inf"))
        out[:, h] = torch.softmax(s, -1) @ v[:, h]
    return out, b.out[first + torch.tensor(rows, device="cuda")].double().view_as(out)


@pytest.mark.parametrize("dtype,H,KH,prefix,lens,rows,takes", [
    ("bf16", 1, 1, 560000, [70], None, "cut"), ("f32", 1, 1, 300000, [70], None, "cut"),
    ("bf16", 8, 8, 5000, [3000], [3000], "tile in 4"), ("bf16", 8, 2, 9000, [40, 2500], [40, 1500], "tile in 4"),
    ("bf16", 20, 20, 4500, [2500], [2500], "tile"), ("bf16", 4, 4, 9000, [40, 100], [4, 6], "cut"),
    ("bf16", 4, 4, 130, [20000, 5], None, "cut"), ("bf16", 20, 20, 0, [700, 3000], [700, 3000], "tile")])
def test_long_contexts(dtype, H, KH, prefix, lens, rows, takes):
    """Chains of more than 64 pages (page ids come 64 at a time) and the longest prefixes, against float64 on the
    GPU at some rows; norms as above, single values within 2^-7 of the largest (two roundings of 2^-8)."""
    b = Batch(dtype, H, KH, prefix, lens, rows, layers=1).gpu()
    assert kernel(b) == takes
    print(f"long contexts: {dtype} {H}/{KH} heads, prefix {prefix}, lengths {lens}", flush=True)
    b.call()
    torch.cuda.synchronize()
    for seq in range(len(lens)):
        n = 1 if rows is None else rows[seq]
        ref, got = reference64(b, seq, sorted({0, n // 3, n // 2, max(n - 2, 0), n - 1}))
        assert (got - ref).norm() <= (1e-5 if dtype == "f32" else 2.0 ** -8) * ref.norm(), seq
        assert (got - ref).abs().max() <= (1e-5 if dtype == "f32" else 2.0 ** -7) * ref.abs().max(), seq


def test_a_shared_prefix_gives_what_a_copy_in_every_sequence_gives():
    """The prefix's 128 tokens as shared pages, and as the first two pages of every block table."""
    b = Batch("bf16", 4, 4, 128, [1, 70, 200, 33]).gpu()
    b.call()
    table = np.concatenate([np.tile(b.pre, (4, 1)), b.table], 1)
    pt = ftts.PageTableView(dev(table), dev([n + 128 for n in b.lens]))
    out = torch.empty_like(b.out)
    ws = torch.empty(ftts.shared_attention_workspace_bytes(4, 4, ftts.BF16, 4, 4, 0, table.shape[1]), dtype=torch.uint8,
                     device="cuda")
    ftts.shared_attention(b.qd, b.kv, b.layer, pt, None, out, ws)
    torch.cuda.synchronize()
    b.check()
    rel = (out.float() - b.out.float()).norm() / out.float().norm()
    assert rel <= 2.0 ** -7  # each is within 2^-8 of the exact result


def test_strides_streams_and_repeats():
    """Strided outputs leave their gaps, another stream works, equal calls give equal bits."""
    b = Batch("bf16", 4, 4, 300, [10, 200, 64], packed=True).gpu()
    b.call()
    wide = torch.full((3, 1024), -7.0, device="cuda", dtype=torch.bfloat16)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    ftts.shared_attention(b.qd[:, :256], b.kv, b.layer, b.pt, b.prefix, wide[:, 256:512], b.ws, stream=side)
    side.synchronize()
    assert torch.equal(wide[:, 256:512], b.out) and (wide[:, :256] == -7).all() and (wide[:, 512:] == -7).all()
    b.check()


def test_a_pass_of_all_three_captured_and_replayed():
    """Lengths -> tables -> append -> attention as one graph: two graphs share a workspace, lengths and
    rows change between replays, and each replay equals the eager calls bit for bit."""
    B, H, P, width, T = 5, 4, 90, 6, 160
    rng = np.random.default_rng(4)
    n_pages = 40
    pool = torch.from_numpy(workload.bf16_round(rng.standard_normal((1, n_pages, 2, H, 64, 64)).astype(np.float32))).cuda().bfloat16()
    prefix = ftts.SharedPrefix(dev([39, 38]), P)
    free = dev(rng.permutation(38))
    ws = torch.empty(ftts.shared_attention_workspace_bytes(H, H, ftts.BF16, B, T, P, width), dtype=torch.uint8, device="cuda")

    class State:
        def __init__(self):
            self.kv = ftts.KVCache.over(pool.clone())
            self.added, self.cached = dev(np.zeros(B)), dev(np.zeros(B))
            self.pt = ftts.PageTableView(dev(np.full((B, width), -1)), dev(np.zeros(B)))
            self.cu, self.slots, self.counts = dev(np.zeros(B + 1)), dev(np.zeros(T)), dev(np.zeros(2))
            self.qkv = torch.zeros((T, 3 * H * 64), device="cuda", dtype=torch.bfloat16)
            self.out = torch.zeros((T, H * 64), device="cuda", dtype=torch.bfloat16)

        def run(self):
            d = H * 64
            ftts.build_tables(self.added, free, n_pages, self.pt.block_table, self.cu, self.slots, self.counts,
                              cached=self.cached, seq_lens=self.pt.seq_lens)
            ftts.append_kv(self.qkv[:, d:2 * d], self.qkv[:, 2 * d:], self.slots, self.kv, 0)
            ftts.shared_attention(self.qkv[:, :d], self.kv, 0, self.pt, prefix, self.out, ws, row_offsets=self.cu)

        def load(self, seed):
            r = np.random.default_rng(seed)
            self.added.copy_(dev(r.multinomial(int(r.integers(1, T)), [1 / B] * B)))
            self.qkv.copy_(torch.from_numpy(r.standard_normal(self.qkv.shape).astype(np.float32)))
            self.pt.block_table.fill_(-1)
            self.kv.pool.copy_(pool)
            self.out.fill_(3.0)

    graphs, states = [], [State(), State()]
    for s in states:
        s.load(0)
        s.run()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            s.run()
        graphs.append(g)
    eager = State()
    for k in range(6):
        s, g = states[k % 2], graphs[k % 2]
        s.load(10 + k)
        g.replay()
        eager.load(10 + k)
        eager.run()
        torch.cuda.synchronize()
        for name in ("out", "slots", "cu", "counts"):
            assert torch.equal(getattr(s, name), getattr(eager, name)), (k, name)
        assert torch.equal(s.kv.pool, eager.kv.pool) and torch.equal(s.pt.block_table, eager.pt.block_table)
        # and what it holds is right
        n = int(s.cu[-1])
        q = s.qkv[:, :H * 64].float().cpu().numpy().reshape(T, H, 64)
        ref = paged.shared_attention(q, s.kv.pool[0].float().cpu().numpy(), [39, 38], P, s.pt.block_table.cpu().numpy(),
                                     s.pt.seq_lens.tolist(), s.cu.tolist())
        got = s.out.float().cpu().numpy().reshape(ref.shape)
        assert np.linalg.norm(got[:n] - ref[:n]) <= 2.0 ** -8 * np.linalg.norm(ref[:n]) and (got[n:] == 3.0).all()
