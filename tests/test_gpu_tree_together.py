"""Tables, rotated append, tree attention and commit as one layer of a decoder with rotations uses them, round after round,
against the oracle that keeps each sequence's accepted tokens as a plain list."""
import numpy as np
import pytest

from oracle import tree
from paper_2607_21042_amd import ftts, workload

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def i32(v):
    return torch.tensor(np.ascontiguousarray(v), dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,KH,layout,dim", [(6, 2, ftts.ROTARY_HALVES, 64), (4, 4, ftts.ROTARY_PAIRS, 24)])
def test_rounds_of_drafts(dtype, H, KH, layout, dim):
    rng = np.random.default_rng(H)
    B, width, n_pages, most = 4, 6, 30, 8
    rot = ftts.Rotary(dim, layout, 10000.0, ftts.ROTARY_PARTS, 4.0, 64)
    f, _ = tree.frequencies(dim, 10000.0, tree.PARTS, 4.0, 64.0)
    scale = float(rot.c.scale)
    pool = torch.full((1, n_pages, 2, KH, 64, 64), float("nan"), device="cuda", dtype=TYPES[dtype])
    kv, table = ftts.KVCache.over(pool), torch.full((B, width), -1, device="cuda", dtype=torch.int32)
    free, cached = list(range(n_pages)), i32([0] * B)
    path, counts, nxt, new = i32(np.zeros((B, most))), i32([0] * B), i32([0] * B), i32([0] * B)
    kept = [[] for _ in range(B)]                          # accepted tokens' unrotated (k, v) rows of each sequence
    for turn in range(6):
        sizes = [70, 3, 40, 1] if turn == 0 else rng.integers(1, 30, B).tolist()
        if turn == 0:                                      # a prompt is a chain, all of it accepted
            parents = [list(range(-1, n - 1)) for n in sizes]
        else:
            parents = [[-1] + [int(rng.integers(max(0, i - 5), i)) for i in range(1, n)] for n in sizes]
        T = sum(sizes)
        x = rng.standard_normal((T, (H + 2 * KH) * 64)).astype(np.float32)
        x = x if dtype == "f32" else workload.bf16_round(x)
        xd = torch.from_numpy(x).cuda().to(TYPES[dtype])
        before = cached.tolist()
        offsets, lens, slots, taken = i32([0] * (B + 1)), i32([0] * B), i32([0] * T), i32([0, 0])
        ftts.build_tables(i32(sizes), i32(free), n_pages, table, offsets, slots, taken, cached=cached, seq_lens=lens)
        torch.cuda.synchronize()
        free = free[int(taken[0]):]
        assert int(taken[1]) == 0
        positions = np.concatenate([c + tree.depths(p) for c, p in zip(before, parents)])
        q = torch.empty((T, H * 64), device="cuda", dtype=TYPES[dtype])
        ftts.append_rotated(xd[:, H * 64:(H + KH) * 64], xd[:, (H + KH) * 64:], rot, i32(positions), slots, kv, 0, q=xd[:, :H * 64], q_out=q)
        masks = torch.cat([ftts.tree_masks(p, 2) for p in parents]).cuda()
        pt = ftts.PageTableView(table, lens)
        ws = torch.empty(ftts.tree_attention_workspace_bytes(H, KH, kv.dtype, B, T, 0, width), dtype=torch.uint8, device="cuda")
        out = torch.empty_like(q)
        ftts.tree_attention(q, kv, 0, pt, masks, offsets, out, ws)
        torch.cuda.synchronize()
        print(f"{dtype} {H}/{KH}, turn {turn}: trees of {sizes} behind {before}", flush=True)
        # every row against its path as a plain sequence
        qr = tree.rotate(x[:, :H * 64], positions, dim, layout, f, scale).reshape(T, H, 64)
        kr, r0 = tree.rotate(x[:, H * 64:(H + KH) * 64], positions, dim, layout, f, scale), 0
        half = 0 if dtype == "f32" else 2.0 ** -8
        for b, up in enumerate(parents):
            old = [tree.rotate(k[None], np.array([t]), dim, layout, f, scale)[0] for t, (k, _) in enumerate(kept[b])]
            for i in sorted({0, len(up) // 2, len(up) - 1}):
                way = [i]
                while up[way[0]] >= 0:
                    way.insert(0, up[way[0]])
                keys = np.array(old + [kr[r0 + j] for j in way]).reshape(-1, KH, 64)
                vals = np.array([v for _, v in kept[b]] + [x[r0 + j, (H + KH) * 64:] for j in way], dtype=np.float64).reshape(-1, KH, 64)
                for h in range(H):
                    s = keys[:, h * KH // H] @ qr[r0 + i, h] / 8
                    p = np.exp(s - s.max())
                    want, size = p @ vals[:, h * KH // H] / p.sum(), p @ np.abs(vals[:, h * KH // H]) / p.sum()
                    got = out[r0 + i, h * 64:(h + 1) * 64].double().cpu().numpy()
                    # queries and keys are rounded to bf16 in the cache (half a step each: scores move by up to `half` twice
                    # their terms' sum), the output once
                    moved = 2 * half * (np.abs(keys[:, h * KH // H]) @ np.abs(qr[r0 + i, h])).max() / 8 + 2.0 ** -17
                    assert (np.abs(got - want) <= np.expm1(2 * moved) * 2 * size + half * np.abs(want) + 1e-5 * size).all(), (turn, b, i, h)
            r0 += len(up)
        tokens = np.concatenate([rng.permutation(50000)[:n] for n in sizes])
        choices, r0, want = rng.integers(50000, 60000, T), 0, []
        for b, up in enumerate(parents):                   # a random way down, as far as it goes
            at, way = 0, [0]
            while len(way) < most and turn:
                below = [j for j in range(len(up)) if up[j] == at]
                if not below or rng.random() < 0.2:
                    break
                choices[r0 + at], at = tokens[r0 + (j := below[int(rng.integers(len(below)))])], j
                way.append(at)
            want.append(way)
            r0 += len(up)
        if turn == 0:                                      # the whole prompt is kept as it lies
            way = [list(range(n)) for n in sizes]
            for b, r in enumerate(np.cumsum([0] + sizes[:-1])):
                kept[b] += [(x[r + j, H * 64:(H + KH) * 64], x[r + j, (H + KH) * 64:]) for j in way[b]]
            cached = lens.clone()
            continue
        ftts.tree_commit(i32(tokens), i32(np.concatenate(parents)), i32(choices), offsets, pt, kv, path, counts, nxt, new)
        torch.cuda.synchronize()
        r0 = 0
        for b, way in enumerate(want):
            assert path[b].tolist()[:len(way)] == way and int(counts[b]) == len(way) and int(nxt[b]) == choices[r0 + way[-1]]
            kept[b] += [(x[r0 + j, H * 64:(H + KH) * 64], x[r0 + j, (H + KH) * 64:]) for j in way]
            r0 += sizes[b]
        cached = new.clone()
        # pages behind the kept tokens go back
        for b, n in enumerate(cached.tolist()):
            free += [int(p) for p in table[b, -(-n // 64):].tolist() if p >= 0]
        assert [len(k) for k in kept] == cached.tolist()
    # the cache holds every accepted token at its place
    bits = pool.double().cpu().numpy()[0]
    for b in range(B):
        for t, (k, v) in enumerate(kept[b]):
            page = int(table[b, t // 64])
            key = tree.rotate(k[None], np.array([t]), dim, layout, f, scale)[0]
            got = bits[page, 0, :, t % 64].reshape(-1)
            assert (np.abs(got - key) <= half * np.abs(key) + 1e-5).all() and np.array_equal(bits[page, 1, :, t % 64].reshape(-1), v.astype(np.float64))
