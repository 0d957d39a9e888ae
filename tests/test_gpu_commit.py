"""The commit of drafted trees against the numpy oracle: paths, counts and moved rows are compared bit for bit."""
import numpy as np
import pytest

from oracle import tree
from paper_2607_21042_amd import ftts, workload

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def dev(a, dtype=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda().to(dtype)


class Drafts:
    """Trees of rows[b] tokens behind past[b] cached ones, and choices that follow a path through each as far as they go;
    `plan(rng, n)` gives a tree's parents, tokens and choices."""

    def __init__(self, dtype, layers, KH, past, rows, plan, most, width=None, before=0, seed=0):
        rng = np.random.default_rng([seed, layers, KH])
        self.dtype, self.most, self.past, self.rows = dtype, most, list(past), list(rows)
        self.lens = [p + n for p, n in zip(past, rows)]
        need = [-(-max(n, 0) // 64) for n in self.lens]
        self.table = np.full((len(rows), width or max(max(need), 1)), -1, dtype=np.int64)
        ids = rng.permutation(sum(need) + 2)
        at = 0
        for b, n in enumerate(need):
            k = min(n, self.table.shape[1])
            self.table[b, :k] = ids[at:at + k]
            at += n
        self.pool = workload.bf16_round(rng.standard_normal((layers, sum(need) + 2, 2, KH, 64, 64)).astype(np.float32))
        self.cu = np.concatenate([[0], np.cumsum(rows)]) + before
        parts = [plan(rng, n) for n in rows]
        pad = [rng.integers(-5, 5, before)]
        self.parents, self.tokens, self.choices = (np.concatenate(pad + [np.array(p[i], dtype=np.int64) for p in parts]) for i in range(3))

    def gpu(self):
        B = len(self.rows)
        self.kv = ftts.KVCache.over(dev(self.pool, TYPES[self.dtype]))
        self.pt = ftts.PageTableView(dev(self.table), dev(self.lens))
        self.dev = [dev(x) for x in (self.tokens, self.parents, self.choices, self.cu)]
        self.out = [torch.full((B, self.most), -7, device="cuda", dtype=torch.int32)]
        self.out += [torch.full((B,), -7, device="cuda", dtype=torch.int32) for _ in range(3)]
        return self

    def call(self, **kw):
        ftts.tree_commit(*self.dev, self.pt, self.kv, *self.out, **kw)
        torch.cuda.synchronize()

    def check(self):
        want = tree.commit(self.tokens, self.parents, self.choices, self.cu, self.table, self.lens, self.pool, self.most)
        for got, w, name in zip(self.out, want, ("path", "counts", "next", "new_lens")):
            assert np.array_equal(got.cpu().numpy(), w), (name, got, w)
        assert np.array_equal(self.kv.pool.float().cpu().numpy(), want[4])
        return want


def random_plan(vocab, reach):
    """Few token values, so that siblings are often alike and choices often match."""
    def plan(rng, n):
        up = [-1] + [int(rng.integers(max(0, i - reach), i)) for i in range(1, n)]
        return up[:n], rng.integers(0, vocab, n), rng.integers(-1, vocab, n)
    return plan


def chain_plan(step, kept):
    """Every step-th token one behind the other, all of them chosen up to `kept`."""
    def plan(rng, n):
        up, tokens, choices = [-1] * n, list(range(100, 100 + n)), [5] * n
        last = 0
        for k, i in enumerate(range(step, n, step)):
            up[i] = last
            if k + 1 < kept:
                choices[last] = tokens[i]
            last = i
        return up, tokens, choices
    return plan


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layers,KH", [(1, 1), (3, 5), (24, 20)])
@pytest.mark.parametrize("vocab,reach", [(2, 3), (3, 12), (5, 40)])
def test_random_trees(dtype, layers, KH, vocab, reach):
    for seed, (past, rows, most) in enumerate((([0], [1], 1), ([60], [16], 4), ([0, 100, 5, 63], [40, 0, 64, 9], 8), ([10, 3, 130], [256, 70, 129], 256))):
        if layers > 3 and sum(rows) > 130:
            rows = [n // 3 for n in rows]
        d = Drafts(dtype, layers, KH, past, rows, random_plan(vocab, reach), most, before=seed, seed=seed).gpu()
        print(f"commit: {dtype} {layers} layers, {KH} heads, rows {rows}", flush=True)
        d.call()
        d.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("step", [1, 2, 3, 5, 30])
@pytest.mark.parametrize("past", [0, 1, 50, 63, 64])
def test_long_paths(dtype, step, past):
    """Paths of up to 256 tokens, moved over pages' ends and over each other's old places."""
    d = Drafts(dtype, 2, 3, [past, 7], [256, 11], chain_plan(step, 1000), 256).gpu()
    print(f"long path: {dtype}, step {step}, past {past}", flush=True)
    d.call()
    want = d.check()
    assert want[1].tolist() == [-(-256 // step), -(-11 // step)]
    for kept in (1, 4, 9):
        d = Drafts(dtype, 2, 3, [past, 7], [256, 11], chain_plan(step, kept), 6).gpu()
        d.call()
        d.check()


def test_many_sequences():
    rng = np.random.default_rng(9)
    rows = rng.integers(0, 40, 64).tolist()
    d = Drafts("bf16", 4, 3, rng.integers(0, 200, 64).tolist(), rows, random_plan(2, 4), 12).gpu()
    d.call()
    d.check()


def test_sequences_that_keep_nothing_and_pages_outside_the_pool():
    d = Drafts("bf16", 2, 2, [100, 20, 5, 60, 150], [3, 4, 6, 40, 9], chain_plan(2, 9), 8, width=3)
    d.lens[1], d.lens[2] = -3, 5
    d.table[3, 1], d.table[0, 1] = 10 ** 6, -2
    d.gpu().call()
    want = d.check()
    assert want[1].tolist() == [2, 0, 0, 8, 5] and want[3].tolist()[1:3] == [-3, 5]
    d = Drafts("bf16", 2, 2, [60], [40], chain_plan(2, 9), 8, width=1).gpu()        # most of the tree is past the table
    d.call()
    d.check()


def test_trees_past_the_largest():
    """Tokens from the 257th on are never kept."""
    d = Drafts("bf16", 1, 1, [5], [300], chain_plan(50, 9), 8).gpu()
    d.call()
    assert d.check()[0].tolist() == [[0, 50, 100, 150, 200, 250, -1, -1]]
    d = Drafts("bf16", 1, 1, [5], [300], chain_plan(64, 9), 8).gpu()
    d.call()
    assert d.check()[0].tolist() == [[0, 64, 128, 192, -1, -1, -1, -1]]


def test_parents_that_make_no_tree():
    """Parents behind their children, themselves, outside: never followed, never read past."""
    up = [-1, 1, 0, 5, 10 ** 9, 2, -10 ** 9, 2]
    def plan(rng, n):
        return up, [4] * 8, [4] * 8
    d = Drafts("bf16", 2, 1, [62], [8], plan, 8).gpu()
    d.call()
    assert d.check()[0].tolist() == [[0, 2, 5, -1, -1, -1, -1, -1]]


def test_replayed_from_a_graph():
    d = Drafts("bf16", 3, 4, [40, 10], [30, 50], random_plan(2, 5), 10).gpu()
    fresh = d.kv.pool.clone()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        d.call()
        with torch.cuda.graph(graph, stream=side):
            ftts.tree_commit(*d.dev, d.pt, d.kv, *d.out)
    rng = np.random.default_rng(3)
    for rows in ([30, 50], [1, 79], [80, 0], [44, 3]):
        d.rows, d.cu = rows, np.concatenate([[0], np.cumsum(rows)])
        d.lens = [min(40 + rows[0], 70), min(10 + rows[1], 60)]
        up = [random_plan(2, 5)(rng, n) for n in rows]
        for i, name in enumerate(("parents", "tokens", "choices")):
            x = np.concatenate([np.array(u[i], dtype=np.int64) for u in up])
            setattr(d, name, np.concatenate([x, np.zeros(80 - len(x), dtype=np.int64)]))
        for t, x in zip(d.dev, (d.tokens, d.parents, d.choices, d.cu)):
            t.copy_(dev(x))
        d.pt.seq_lens.copy_(dev(d.lens))
        d.kv.pool.copy_(fresh)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        d.check()


def test_far_pages():
    """Element offsets past 2^31 in a large pool."""
    n_pages = 13200                                    # x 2 x 20 heads x 4096: 1.08e9 elements a layer
    d = Drafts("bf16", 2, 20, [55], [30], chain_plan(3, 9), 12).gpu()
    pool = torch.zeros((2, n_pages, 2, 20, 64, 64), device="cuda", dtype=torch.bfloat16)
    far, ids = [n_pages - 1, n_pages - 2], d.table[0, :2].tolist()
    pool[:, far] = d.kv.pool[:, ids]
    near = d.kv
    d.call()
    d.check()
    d.kv, d.pt = ftts.KVCache.over(pool), ftts.PageTableView(dev([far]), dev(d.lens))
    d.call()
    assert torch.equal(pool[:, far], near.pool[:, ids]) and not pool[:, :n_pages - 2].any()
