"""Every form in which ftts_tree_attention is launched (ftts_tree_attention_plan says which a call takes): 4 and 8 waves, one
part and several, waves with more half pages than they list at once (64), of chains that repeat a few physical pages.

Bounds as in tests/test_gpu_tree.py (u = 2^-24; scores off by 82 u times the largest sum_d |q_d k_d| / 8, the exponential
by 8 u more, a mean over n tokens by 2 (n + 16) u of sum p |v| / sum p, in bf16 2^-16 of that and one rounding of the output).
Over a whole output the roundings of n sums are independent, sqrt(n) u, and those of the output a norm of 2^-8 / sqrt(3).
"""
import numpy as np
import pytest

from oracle import tree
from paper_2607_21042_amd import ftts, workload
from tests.test_gpu_tree import TYPES, U, Trees, dev, random_tree

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
LISTED = 64    # half pages that a wave lists at once


def over(least, most, B, *first):
    """Sizes of B sequences: the first ones as given, the rest spread over [least, most]."""
    return list(first) + [least + i * (most - least) // max(B - len(first) - 1, 1) for i in range(B - len(first))]


# dtype, heads, key heads, own tokens before each tree, trees, prefix, table's width: waves, parts, half pages of the longest wave
FORMS = [
    ("bf16", 20, 20, over(0, 900, 48, 128 * 64 - 10, 8300, 8250), over(1, 1, 48, 40, 20, 3), 0, 131, (4, 1, 66)),
    ("f32", 20, 20, over(0, 900, 48, 128 * 64 - 10, 8300, 8250), over(1, 1, 48, 40, 20, 3), 0, 131, (4, 1, 66)),
    ("bf16", 8, 1, [255 * 64 - 50, 16450, 300, 0, 16500, 70], [256] * 6, 0, 262, (8, 1, 66)),
    ("f32", 8, 1, [255 * 64 - 50, 16450, 300, 0, 16500, 70], [256] * 6, 0, 262, (8, 1, 66)),
    ("bf16", 20, 20, over(0, 700, 32, 16500, 129 * 64 - 90, 127 * 64 - 20), over(1, 1, 32, 19, 11, 1), 70, 260, (4, 2, 66)),
    ("bf16", 20, 20, over(0, 400, 16, 12700, 9000, 64), over(1, 1, 16, 20, 16, 1), 20000, 200, (4, 4, 65)),
    ("f32", 20, 20, over(0, 400, 16, 12700, 9000, 64), over(1, 1, 16, 20, 16, 1), 20000, 200, (8, 2, 65)),
    ("f32", 20, 20, over(0, 400, 12, 13400, 9000, 64), over(1, 1, 12, 14, 6, 1), 20000, 210, (4, 4, 66)),
    ("bf16", 1, 1, [100, 3], [6, 2], 20000, 2, (8, 48, 2)),
    ("bf16", 1, 1, [18900], [256], 0, 300, (8, 24, 4)),
    ("bf16", 4, 2, [2400, 100], [70, 30], 0, 40, (4, 8, 3)),
    ("f32", 4, 2, [2400, 100], [70, 30], 0, 40, (4, 12, 2)),
    ("f32", 20, 4, over(0, 6700, 8), [62] * 8, 0, 106, (8, 2, 14)),
]


class Long(Trees):
    """As Trees, but that the prefix and the own pages before a tree are drawn from a few physical ones, each with values
    about a mean of its own; a tree's pages are its sequence's alone, NaN behind its last token."""

    def __init__(self, dtype, H, KH, past, rows, prefix, width, stock=13, seed=0):
        rng = np.random.default_rng([seed, prefix, H])
        self.dtype, self.H, self.KH, self.P, self.rows, self.past = dtype, H, KH, prefix, list(rows), list(past)
        self.lens, self.width, self.layer = [p + n for p, n in zip(past, rows)], width, 0
        first, last = [p // 64 for p in past], [-(-n // 64) for n in self.lens]
        n_pages = stock + sum(hi - lo for lo, hi in zip(first, last))
        self.pre = rng.integers(0, stock, -(-prefix // 64))
        self.table = np.full((len(rows), width), -1, dtype=np.int64)
        pool = rng.standard_normal((1, n_pages, 2, KH, 64, 64)).astype(np.float32) * np.float32(0.7)
        pool[:, :, 1] += rng.standard_normal((n_pages, KH, 1, 64)).astype(np.float32)
        at = stock
        for b, (lo, hi) in enumerate(zip(first, last)):
            self.table[b, :lo] = rng.integers(0, stock, lo)
            self.table[b, lo:hi] = at + np.arange(hi - lo)
            at += hi - lo
            if self.lens[b] % 64:
                pool[0, at - 1, :, :, self.lens[b] % 64:] = np.nan
        self.pool = pool if dtype == "f32" else workload.bf16_round(pool)
        self.cu = np.concatenate([[0], np.cumsum(rows)])
        self.T, self.words = int(self.cu[-1]), -(-max(rows) // 64)
        self.parents = [random_tree(rng, n) for n in rows]
        self.masks = np.concatenate([tree.masks(up, self.words) for up in self.parents])
        q = rng.standard_normal((self.T, H * 64)).astype(np.float32) * np.float32(0.7)
        self.q = q if dtype == "f32" else workload.bf16_round(q)

    def near(self):
        lim = 0.0 if self.dtype == "f32" else 2.0 ** -8
        for b, n in enumerate(self.rows):
            r0, past, G = int(self.cu[b]), self.past[b], self.H // self.KH
            ids = np.concatenate([self.pre, self.table[b, :-(-self.lens[b] // 64)]])
            at = np.concatenate([np.arange(self.P), -(-self.P // 64) * 64 + np.arange(self.lens[b])])
            kv = self.kv.pool[0][dev(ids).long()].double()
            k, v = (kv[:, j].permute(1, 0, 2, 3).reshape(self.KH, -1, 64)[:, dev(at).long()] for j in (0, 1))
            seen = np.ones((n, self.P + past + n), dtype=bool)
            bits = self.masks[r0:r0 + n].view(np.uint64)
            for j in range(n):
                seen[:, self.P + past + j] = (bits[:, j // 64] >> np.uint64(j % 64) & np.uint64(1)).astype(bool)
            seen = dev(seen, torch.bool).repeat(G, 1)
            q = self.qd[r0:r0 + n].double().view(n, self.KH, G, 64).permute(1, 2, 0, 3).reshape(self.KH, G * n, 64)
            p = torch.softmax((q @ k.transpose(1, 2) / 8).masked_fill_(~seen, -np.inf), -1)
            ref, size = p @ v, p @ v.abs()
            dots = (q.abs() @ k.abs().transpose(1, 2) / 8).masked_fill_(~seen, 0).amax(-1, keepdim=True)
            got = self.out[r0:r0 + n].double().view(n, self.KH, G, 64).permute(1, 2, 0, 3).reshape(ref.shape)
            eps, err, count = 82 * U * dots + 8 * U, (got - ref).abs(), seen.shape[1]
            half = 2.0 ** -16 if lim else 0.0
            bound = (2 * eps + 2 * U * (count + 16) + half) * size
            assert torch.isfinite(err).all() and (err <= bound + lim * (ref.abs() + bound)).all(), (b, (err - bound).max())
            norm = ((2 * eps + 2 * U * count ** 0.5 + half) * size).norm() + lim / 3 ** 0.5 * ref.norm()
            assert err.norm() <= norm, (b, err.norm().item(), norm.item())


def name(f):
    return f"{f[0]} {f[1]}/{f[2]} heads, {len(f[3])} sequences, prefix {f[5]}, width {f[6]}: {f[7]}"


def taken(dtype, H, KH, past, rows, prefix, width):
    p = ftts.tree_attention_plan(H, KH, ftts.F32 if dtype == "f32" else ftts.BF16, len(rows), sum(rows), prefix, width)
    each = -(-(-(-prefix // 64) + width) // p.parts)
    return p.waves, p.parts, -(-2 * each // p.waves)


@pytest.mark.parametrize("form", FORMS, ids=name)
def test_forms(form):
    assert taken(*form[:7]) == form[7]
    t = Long(*form[:7]).gpu()
    print(name(form), flush=True)
    t.call()
    t.near()
    again = t.out.clone()
    t.ws.fill_(0xFF)
    t.call()
    assert torch.equal(t.out, again)


@pytest.mark.parametrize("form", [f for f in FORMS if len(f[3]) <= 8], ids=name)
def test_values_that_are_not_finite(form):
    """NaN and infinities at a tree's tokens reach those tokens' descendants and no one else, in every form."""
    t = Long(*form[:7]).gpu()
    print(f"not finite: {name(form)}", flush=True)
    t.call()
    clean, fresh = t.out.clone(), t.kv.pool.clone()
    n, past = t.rows[0], t.past[0]
    for node in (1, n // 2, n - 1):
        sees = torch.zeros(t.T, dtype=torch.bool, device="cuda")
        sees[:n] = dev(t.masks[:n, node // 64] >> (node % 64) & 1, torch.bool)
        at = past + node
        for kv, what in ((1, np.nan), (1, np.inf), (1, -np.inf), (0, np.nan), (0, np.inf)):
            t.kv.pool.copy_(fresh)
            t.kv.pool[0, int(t.table[0, at // 64]), kv, :, at % 64] = what
            t.call()
            assert torch.equal(t.out[~sees], clean[~sees]), (node, kv, what)
            got = t.out[sees].float()
            if kv == 1:
                assert (torch.isnan(got) if np.isnan(what) else got == what).all(), (node, what)
            else:
                assert torch.isnan(got).all() or np.isinf(what), (node, what)
