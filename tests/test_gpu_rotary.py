"""Rows turned by their positions, and keys and values turned into their pages, against the numpy oracle (float64).

With u = 2^-24: cosine and sine take an angle that is off by 2^-28 turns at most (0.4 u) and are off by 2 steps (4 u)
more; the factor, the product that is rounded by itself and the sum add u each, so an fp32 result is off by at most
8 u s (|a| + |b|) for a pair (a, b) and factor s.  A bf16 result is rounded once more, 2^-8 of itself.
"""
import numpy as np
import pytest

from oracle import paged, tree
from paper_2607_21042_amd import ftts, workload

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
U = 2.0 ** -24
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def dev(a, dtype=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda().to(dtype)


def rows(rng, shape, src):
    x = rng.standard_normal(shape).astype(np.float32)
    return workload.bf16_round(x) if src == "bf16" else x


def check(got, x, positions, dim, layout, f, scale, dst, what):
    want = tree.rotate(x, positions, dim, layout, f, scale)
    size = np.abs(x.astype(np.float64)).reshape(len(x), -1, 64)
    h = dim // 2
    a, b = (slice(0, h), slice(h, dim)) if layout == tree.HALVES else (slice(0, dim, 2), slice(1, dim, 2))
    both = np.zeros_like(size)
    both[..., a] = both[..., b] = abs(scale) * (size[..., a] + size[..., b])
    tol = 8 * U * both.reshape(x.shape)
    if dst == "bf16":
        tol = tol * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(want)
    bad = np.abs(got - want) > tol
    assert not bad.any(), (what, np.argwhere(bad)[:4], got[bad][:4], want[bad][:4])
    left, keep = got.reshape(len(x), -1, 64)[..., dim:], x.reshape(len(x), -1, 64)[..., dim:]
    assert np.array_equal(left, workload.bf16_round(np.ascontiguousarray(keep)) if dst == "bf16" else keep), what


FORMS = [(tree.HALVES, 64), (tree.HALVES, 32), (tree.HALVES, 48), (tree.HALVES, 20), (tree.HALVES, 62), (tree.HALVES, 2),
         (tree.PAIRS, 64), (tree.PAIRS, 24), (tree.PAIRS, 2), (tree.PAIRS, 38)]


@pytest.mark.parametrize("src,dst", [("bf16", "bf16"), ("f32", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("layout,dim", FORMS)
def test_rotate(src, dst, layout, dim):
    for T, H, pad, scaling in ((1, 1, 0, tree.PLAIN), (5, 3, 64, tree.LINEAR), (67, 20, 2560, tree.PARTS), (2100, 5, 8, tree.BASE)):
        if scaling == tree.BASE and dim == 2:
            continue
        rng = np.random.default_rng([T, dim, layout])
        print(f"rotate: {src} -> {dst}, layout {layout}, {dim} columns, {T} rows, {H} heads", flush=True)
        x = rows(rng, (T, H * 64 + pad), src)
        pos = rng.integers(-2 ** 20, 2 ** 20, T)
        pos[:: 7] = rng.choice([0, 1, 2 ** 31 - 1, -2 ** 31], len(pos[:: 7])) if T > 1 else 3
        f, scale = tree.frequencies(dim, 10000.0, scaling, 8.0, 512.0)
        rot = ftts.Rotary(dim, layout, 10000.0, scaling, 8.0, 512)
        if (abs(pos) > 2 ** 21).any():
            # far positions: the reference takes the library's own turns, in 64 bits a position of 2^31 shows their last step
            f = np.array(rot.turns) * (2 * np.pi)
        out = torch.full((T, H * 64), 9.0, device="cuda", dtype=TYPES[dst])
        xs = dev(x, TYPES[src])
        ftts.rotate(xs[:, :H * 64], rot, dev(pos), out)
        torch.cuda.synchronize()
        near = abs(pos) <= 2 ** 21
        got = out.float().cpu().numpy()
        check(got[near], x[near, :H * 64], pos[near], dim, layout, f, float(rot.c.scale), dst, (T, H))
        # at 2^31 the oracle's own angle is off by 2^31 2^-53 radians and more: 2^-20 of |a| + |b| on top
        if (~near).any():
            want = tree.rotate(x[~near, :H * 64], pos[~near], dim, layout, f, float(rot.c.scale))
            assert np.abs(got[~near] - want).max() <= (2.0 ** -7 if dst == "bf16" else 2.0 ** -20) * 2 * rot.c.scale * np.abs(x).max()
        assert torch.equal(xs.float().cpu(), torch.from_numpy(x))


@pytest.mark.parametrize("layout,dim", FORMS)
@pytest.mark.parametrize("t", ["bf16", "f32"])
def test_rotate_in_place_and_into_other_columns(layout, dim, t):
    rng = np.random.default_rng(dim)
    for T in (1, 40, 3000):
        x = rows(rng, (T, 3 * 256), t)
        pos = rng.integers(0, 5000, T)
        rot = ftts.Rotary(dim, layout)
        print(f"in place: {t}, layout {layout}, {dim} columns, {T} rows", flush=True)
        a = dev(x, TYPES[t])
        ftts.rotate(a[:, :256], rot, dev(pos), a[:, 512:])
        b = dev(x, TYPES[t])
        ftts.rotate(b[:, :256], rot, dev(pos), b[:, :256])
        torch.cuda.synchronize()
        f, scale = tree.frequencies(dim, 10000.0)
        check(a[:, 512:].float().cpu().numpy(), x[:, :256], pos, dim, layout, f, scale, t, "other columns")
        assert torch.equal(a[:, 512:], b[:, :256])
        assert torch.equal(a[:, :512].float().cpu(), torch.from_numpy(x[:, :512])) and torch.equal(b[:, 256:].float().cpu(), torch.from_numpy(x[:, 256:]))


def test_values_that_are_not_finite_stay_in_their_pair():
    for layout, dim in FORMS:
        x = torch.ones((1, 128), device="cuda")
        x[0, 0], x[0, 64 + dim - 1], x[0, 63] = float("inf"), float("nan"), float("-inf") if dim < 64 else 1.0
        out = torch.zeros_like(x)
        ftts.rotate(x, ftts.Rotary(dim, layout), dev([3]), out)
        torch.cuda.synchronize()
        h = dim // 2
        pair = {0, h} if layout == tree.HALVES else {0, 1}
        last = {64 + h - 1, 64 + dim - 1} if layout == tree.HALVES else {64 + dim - 2, 64 + dim - 1}
        odd = set(torch.nonzero(~torch.isfinite(out[0])).flatten().tolist())
        assert odd == pair | last | ({63} if dim < 64 else set()), (layout, dim, odd)


@pytest.mark.parametrize("src,dst", [("bf16", "bf16"), ("f32", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("T,H,KH,packed", [(1, 1, 1, False), (3, 8, 4, True), (64, 20, 20, True), (130, 12, 2, False), (257, 0, 5, True),
                                           (2500, 4, 1, True)])
@pytest.mark.parametrize("layout,dim", [(tree.HALVES, 64), (tree.HALVES, 36), (tree.PAIRS, 64), (tree.PAIRS, 18)])
def test_append(src, dst, T, H, KH, packed, layout, dim):
    rng = np.random.default_rng([T, H, KH])
    n_pages, a, b = T // 64 + 3, H * 64, KH * 64
    x = rows(rng, (T, a + 2 * b + (0 if packed else 16)), src)
    slots = rng.permutation(n_pages * 64)[:T]
    slots[::5] = rng.choice([-1, -70, n_pages * 64, 2 ** 31 - 1], len(slots[::5])) if T > 1 else slots[::5]
    pos = rng.integers(0, 2 ** 20, T)
    old = workload.bf16_round(rng.standard_normal((2, n_pages, 2, KH, 64, 64)).astype(np.float32))
    xs, pool = dev(x, TYPES[src]), dev(old, TYPES[dst])
    rot = ftts.Rotary(dim, layout, 500000.0, ftts.ROTARY_PARTS, 8.0, 4096)
    f, _ = tree.frequencies(dim, 500000.0, tree.PARTS, 8.0, 4096.0)
    scale = float(rot.c.scale)
    q_out = torch.full((T, a), 7.0, device="cuda", dtype=TYPES[dst]) if H else None
    print(f"append: {src} -> {dst}, {T} rows, {H}/{KH} heads, layout {layout}, {dim} columns", flush=True)
    ftts.append_rotated(xs[:, a:a + b], xs[:, a + b:a + 2 * b], rot, dev(pos), dev(slots), ftts.KVCache.over(pool), 1,
                        q=xs[:, :a] if H else None, q_out=q_out)
    torch.cuda.synchronize()
    got, kept = pool.float().cpu().numpy(), (slots >= 0) & (slots < n_pages * 64)
    v = workload.bf16_round(x) if dst == "bf16" else x
    want = paged.append(old, 1, np.zeros((T, b), np.float32), v[:, a + b:a + 2 * b], slots)
    page, at = slots[kept] // 64, slots[kept] % 64
    keys = got[1, page, 0, :, at].reshape(-1, b)
    check(keys, np.ascontiguousarray(x[kept, a:a + b]), pos[kept], dim, layout, f, scale, dst, "keys")
    got[1, page, 0, :, at] = 0
    assert np.array_equal(got, want)
    if H:
        q = q_out.float().cpu().numpy()
        check(q[kept], np.ascontiguousarray(x[kept, :a]), pos[kept], dim, layout, f, scale, dst, "queries")
        assert (q[~kept] == 7).all()


def test_append_equals_rotate_and_append():
    """Bit for bit, queries in place, on a stream of its own, replayed from a graph with new positions."""
    rng = np.random.default_rng(5)
    T, H, KH = 70, 20, 4
    x = dev(rng.standard_normal((T, (H + 2 * KH) * 64)).astype(np.float32), torch.bfloat16)
    slots, rot = dev(rng.permutation(256)[:T]), ftts.Rotary(32, ftts.ROTARY_PAIRS)
    pos = dev(rng.integers(0, 1000, T))
    a, b = H * 64, KH * 64

    def pools():
        return [torch.zeros((1, 4, 2, KH, 64, 64), device="cuda", dtype=torch.bfloat16) for _ in range(2)]
    side = torch.cuda.Stream()
    ours, theirs = pools()
    work, src = x.clone(), x.clone()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        def step():
            work.copy_(src)
            ftts.append_rotated(work[:, a:a + b], work[:, a + b:], rot, pos, slots, ftts.KVCache.over(ours), 0, q=work[:, :a],
                                q_out=work[:, :a])
        step()
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            step()
    for k in range(4):
        pos.copy_(dev(rng.integers(0, 2 ** 20, T)))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        k_rot, q_rot = torch.empty((T, b), device="cuda", dtype=torch.bfloat16), torch.empty((T, a), device="cuda", dtype=torch.bfloat16)
        ftts.rotate(x[:, a:a + b], rot, pos, k_rot)
        ftts.rotate(x[:, :a], rot, pos, q_rot)
        ftts.append_kv(k_rot, x[:, a + b:].contiguous(), slots, ftts.KVCache.over(theirs), 0)
        torch.cuda.synchronize()
        assert torch.equal(ours, theirs) and torch.equal(work[:, :a], q_rot) and torch.equal(work[:, a:], x[:, a:])


@pytest.mark.parametrize("T,H", [(1, 256), (9, 100), (700, 256), (4097, 20)])
@pytest.mark.parametrize("layout,dim", [(tree.HALVES, 64), (tree.HALVES, 20), (tree.PAIRS, 64)])
def test_many_heads_in_place(T, H, layout, dim):
    rng = np.random.default_rng([T, H])
    x = rows(rng, (T, H * 64), "bf16")
    pos = rng.integers(0, 5000, T)
    f, scale = tree.frequencies(dim, 10000.0)
    print(f"in place: {T} rows of {H} heads, layout {layout}, {dim} columns", flush=True)
    a = dev(x, torch.bfloat16)
    ftts.rotate(a, ftts.Rotary(dim, layout), dev(pos), a)
    torch.cuda.synchronize()
    some = sorted({0, T // 2, T - 1} | set(rng.integers(0, T, 40).tolist()))
    check(a[some].float().cpu().numpy(), x[some], pos[some], dim, layout, f, scale, "bf16", (T, H))


def test_far_pages():
    """Element offsets past 2^31 in a large pool."""
    n_pages, T = 13200, 70                             # x 2 x 20 heads x 4096: 1.08e9 elements a layer
    pool = torch.zeros((2, n_pages, 2, 20, 64, 64), device="cuda", dtype=torch.bfloat16)
    near = torch.zeros((1, 2, 2, 20, 64, 64), device="cuda", dtype=torch.bfloat16)
    x = dev(rows(np.random.default_rng(1), (T, 40 * 64), "bf16"), torch.bfloat16)
    rot, pos = ftts.Rotary(64), dev(np.arange(T) * 13)
    ftts.append_rotated(x[:, :1280], x[:, 1280:], rot, pos, dev(np.arange(T)), ftts.KVCache.over(near), 0)
    ftts.append_rotated(x[:, :1280], x[:, 1280:], rot, pos, dev((n_pages - 2) * 64 + np.arange(T)), ftts.KVCache.over(pool), 1)
    torch.cuda.synchronize()
    assert torch.equal(pool[1, n_pages - 2:], near[0]) and not pool[0].any() and not pool[1, :n_pages - 2].any()
