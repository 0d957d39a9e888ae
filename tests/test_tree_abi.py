"""Refusals of the entry points for drafted trees, without a GPU (every call fails before anything is enqueued)."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import tree
from paper_2607_21042_amd import ftts

FAKE = 0x100000
L = ftts.lib()


def shape(dtype=1, heads=20, kvh=20, d=64):
    return ftts.AttnShape(dtype, heads, kvh, d)


def attend(sh=None, q=FAKE, qs=1280, cu=FAKE, rows=40, B=4, masks=FAKE, words=1, prefix=None, table=FAKE, lens=FAKE, width=8, base=FAKE,
           pages=9, layer=0, out=FAKE * 2, outs=1280, ws=FAKE, size=1 << 30, pt=True):
    t, kv = ftts.PageTable(table, lens, width), ftts.KvPool(base, pages)
    return L.ftts_tree_attention(None if sh == 0 else ctypes.byref(sh or shape()), q, qs, cu, rows, B, masks, words,
                                 ctypes.byref(prefix) if prefix else None, ctypes.byref(t) if pt else None, ctypes.byref(kv), layer, out,
                                 outs, ws, size, None)


@pytest.mark.parametrize("bad,code", [
    (dict(sh=0), -1), (dict(sh=shape(dtype=2)), -3), (dict(sh=shape(d=32)), -7), (dict(sh=shape(heads=0)), -2),
    (dict(sh=shape(heads=257, kvh=1)), -2), (dict(sh=shape(kvh=3)), -2), (dict(B=0), -2), (dict(B=65), -2), (dict(rows=-1), -5),
    (dict(rows=(1 << 24) + 1), -5), (dict(sh=shape(heads=256, kvh=1), qs=16384, outs=16384, rows=1 << 23), -5), (dict(words=0), -2),
    (dict(words=5), -2), (dict(masks=None), -1), (dict(masks=FAKE + 4), -4), (dict(cu=None), -1), (dict(q=None), -1), (dict(out=None), -1),
    (dict(qs=1276), -2), (dict(outs=1284), -2), (dict(qs=1216), -2), (dict(q=FAKE + 8), -4), (dict(out=FAKE + 2), -4),
    (dict(base=FAKE + 8), -4), (dict(base=None), -1), (dict(pages=0), -2), (dict(layer=-1), -2), (dict(width=0), -2), (dict(width=513), -2),
    (dict(table=None), -1), (dict(lens=None), -1), (dict(pt=False), -1), (dict(ws=None), -1), (dict(ws=FAKE + 4), -4), (dict(size=16), -8),
    (dict(prefix=ftts.SharedPrefixC(None, 5)), -1), (dict(prefix=ftts.SharedPrefixC(FAKE, -1)), -5),
    (dict(prefix=ftts.SharedPrefixC(FAKE, (1 << 20) + 1)), -5)])
def test_attention_refused(bad, code):
    assert attend(**bad) == code, L.ftts_last_error()


def test_attention_of_nothing():
    assert attend(rows=0) == 0 and attend(rows=0, q=None, out=None, masks=None, ws=None) == 0


def test_workspaces_cover_smaller_calls():
    size = lambda *a, **k: L.ftts_tree_attention_workspace_bytes(ctypes.byref(shape(**k)), *a)  # noqa: E731
    assert size(0, 5, 0, 4) == 0 and size(4, 5, -1, 4) == 0 and size(4, 5, 0, 0) == 0 and size(4, -1, 0, 4) == 0
    rng = np.random.default_rng(0)
    for _ in range(300):
        heads, kvh = [(20, 20), (20, 4), (8, 1), (1, 1), (256, 8)][rng.integers(5)]
        big = [int(rng.integers(1, 65)), int(rng.integers(0, 5000)), int(rng.integers(0, 20000)), int(rng.integers(1, 513))]
        small = [int(rng.integers(1, big[0] + 1)), int(rng.integers(0, big[1] + 1)), int(rng.integers(0, big[2] + 1)), int(rng.integers(1, big[3] + 1))]
        for dtype in (0, 1):
            assert 0 < size(*small, heads=heads, kvh=kvh, dtype=dtype) <= size(*big, heads=heads, kvh=kvh, dtype=dtype), (small, big)


def test_masks_from_parents():
    rng = np.random.default_rng(1)
    for n in (1, 5, 64, 65, 256):
        up = [-1] + [int(rng.integers(0, i)) for i in range(1, n)]
        got = ftts.tree_masks(up)
        assert got.dtype == torch.int64 and np.array_equal(got.numpy(), tree.masks(up, -(-n // 64)))
    assert ftts.tree_masks([-1, 0], words=3).shape == (2, 3) and ftts.tree_masks([]).shape == (0, 0)
    for bad in ([-1, 1], [-1, -2], [-1, 0, 3]):
        with pytest.raises(ftts.FTTSError):
            ftts.tree_masks(bad)
    with pytest.raises(ftts.FTTSError):
        ftts.tree_masks([-1] * 65, words=1)
    with pytest.raises(ftts.FTTSError):
        ftts.tree_masks([-1] * 257)


def test_binding_refuses_before_the_library():
    def call(q=(3, 128), dtype=torch.bfloat16, out=torch.bfloat16, masks=(3, 1), mtype=torch.int64, layer=0, lens=2, cu=3):
        pool = type("kv", (), {"pool": torch.zeros((1, 2, 2, 2, 64, 64), dtype=torch.bfloat16), "dtype": ftts.BF16, "c": ftts.KvPool()})
        pt = type("pt", (), {"block_table": torch.zeros((2, 2), dtype=torch.int32), "seq_lens": torch.zeros(lens, dtype=torch.int32), "c": ftts.PageTable()})
        ftts.tree_attention(torch.zeros(q, dtype=dtype), pool, layer, pt, torch.zeros(masks, dtype=mtype), torch.zeros(cu, dtype=torch.int32),
                            torch.zeros(q, dtype=out), torch.zeros(16, dtype=torch.uint8))
    for bad, code in ((dict(q=(3, 100)), -2), (dict(dtype=torch.float32), -3), (dict(out=torch.float32), -3), (dict(mtype=torch.int32), -3),
                      (dict(masks=(2, 1)), -2), (dict(masks=(3,)), -2), (dict(layer=1), -5), (dict(lens=1), -2), (dict(cu=2), -2), ({}, -1)):
        with pytest.raises(ftts.FTTSError) as e:
            call(**bad)
        assert e.value.code == code, (bad, e.value)


I = torch.int32


def commit(tokens=FAKE, parents=FAKE * 2, choices=FAKE * 3, cu=FAKE * 4, rows=40, B=4, table=FAKE * 5, lens=FAKE * 6, width=8, base=FAKE * 64,
           pages=9, dtype=1, layers=24, kvh=20, path=FAKE * 7, most=8, counts=FAKE * 8, nxt=FAKE * 9, new=FAKE * 10, pt=True):
    t, kv = ftts.PageTable(table, lens, width), ftts.KvPool(base, pages)
    return L.ftts_tree_commit(tokens, parents, choices, cu, rows, B, ctypes.byref(t) if pt else None, ctypes.byref(kv), dtype, layers, kvh,
                              path, most, counts, nxt, new, None)


@pytest.mark.parametrize("bad,code", [
    (dict(dtype=2), -3), (dict(pt=False), -1), (dict(table=None), -1), (dict(lens=None), -1), (dict(base=None), -1), (dict(B=0), -2),
    (dict(B=65), -2), (dict(rows=-1), -5), (dict(rows=(1 << 24) + 1), -5), (dict(width=0), -2), (dict(width=513), -2), (dict(pages=0), -2),
    (dict(layers=0), -2), (dict(kvh=0), -2), (dict(kvh=257), -2), (dict(layers=1 << 20, kvh=1), -2), (dict(most=0), -2), (dict(most=257), -2),
    (dict(tokens=None), -1), (dict(parents=None), -1), (dict(choices=None), -1), (dict(cu=None), -1), (dict(path=None), -1),
    (dict(counts=None), -1), (dict(nxt=None), -1), (dict(new=None), -1), (dict(base=FAKE * 64 + 8), -4), (dict(path=FAKE * 7 + 1), -4),
    (dict(tokens=FAKE + 2), -4), (dict(new=FAKE * 6), -1), (dict(path=FAKE * 3 + 16), -1), (dict(counts=FAKE * 9 - 8), -1),
    (dict(nxt=FAKE * 64 + 64), -1), (dict(lens=FAKE * 64 + 4096), -1), (dict(counts=FAKE * 5 + 64), -1)])
def test_commit_refused(bad, code):
    assert commit(**bad) == code, L.ftts_last_error()


def test_commit_binding_refuses_before_the_library():
    def call(tokens=5, parents=5, choices=5, cu=3, path=(2, 4), counts=2, lens=2, dtype=I):
        pool = type("kv", (), {"pool": torch.zeros((1, 2, 2, 2, 64, 64), dtype=torch.bfloat16), "dtype": ftts.BF16, "c": ftts.KvPool()})
        pt = type("pt", (), {"block_table": torch.zeros((2, 2), dtype=I), "seq_lens": torch.zeros(lens, dtype=I), "c": ftts.PageTable()})
        z = lambda n: torch.zeros(n, dtype=I)  # noqa: E731
        ftts.tree_commit(torch.zeros(tokens, dtype=dtype), z(parents), z(choices), z(cu), pt, pool, z(path), z(counts), z(2), z(2))
    for bad, code in ((dict(dtype=torch.int64), -3), (dict(parents=4), -2), (dict(choices=6), -2), (dict(cu=2), -2), (dict(path=(3, 4)), -2),
                      (dict(path=(8,)), -2), (dict(counts=3), -2), (dict(lens=3), -2), ({}, -1)):
        with pytest.raises(ftts.FTTSError) as e:
            call(**bad)
        assert e.value.code == code, (bad, e.value)


@pytest.mark.parametrize("heads,kvh,B,most", [(256, 256, 4, 65524 * 32 + 31), (64, 1, 64, ((1 << 24) - 72) // 2), (20, 4, 33, None)])
def test_attention_refuses_more_tiles_than_a_launch_takes(heads, kvh, B, most):
    """Tiles of 32 (row, head) pairs, in blocks of 8 where they are 16 and more: fewer than 2^24 of them, 2^32 threads."""
    def tiles(rows):
        n = rows * (heads // kvh) // 32 + B
        return kvh * (-(-n // 8) * 8 if n >= 16 else n)
    lo, hi = 1, 1 << 24
    while hi - lo > 1:                                     # (lo fits, hi does not)
        mid = (lo + hi) // 2
        lo, hi = (mid, hi) if tiles(mid) < 1 << 24 else (lo, mid)
    assert most in (None, lo) and (tiles(hi) >= 1 << 24 or hi == 1 << 24)
    sh, wide = shape(heads=heads, kvh=kvh), 64 * heads
    size = lambda rows: L.ftts_tree_attention_workspace_bytes(ctypes.byref(sh), B, rows, 0, 4)  # noqa: E731
    assert size(lo) > 0 and attend(sh=sh, rows=lo, B=B, qs=wide, outs=wide, size=16) == -8
    if hi < 1 << 24:
        assert size(hi) == 0 and attend(sh=sh, rows=hi, B=B, qs=wide, outs=wide) == -5
