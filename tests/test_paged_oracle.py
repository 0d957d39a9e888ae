"""Pins of the paged-serving oracle (oracle/paged.py) and the argument checks of its three
operators, which need no GPU: every call below is refused before anything is enqueued."""
import ctypes

import numpy as np
import pytest

from oracle import paged
from paper_2607_21042_amd import ftts

FAKE = 0x100000  # aligned, never dereferenced


# ---- the oracle -----------------------------------------------------------------------------
def test_tables_by_hand():
    old = np.array([[7, 8, 5], [3, 9, 9], [9, 9, 9], [4, 9, 9]])
    #         2 pages kept, 1 new | inside its page | nothing | 2 new
    cached, added = [100, 10, 0, 64], [60, 5, 0, 70]
    table, cu, lens, slots, counts = paged.build_tables(cached, added, [20, 21, 22, 23], 30, old, 140)
    assert table.tolist() == [[7, 8, 20], [3, -1, -1], [-1, -1, -1], [4, 21, 22]]
    assert cu.tolist() == [0, 60, 65, 65, 135] and lens.tolist() == [160, 15, 0, 134]
    assert counts.tolist() == [3, 0]
    assert slots[0] == 8 * 64 + 36 and slots[27] == 8 * 64 + 63 and slots[28] == 20 * 64 and slots[59] == 20 * 64 + 31
    assert slots[60] == 3 * 64 + 10 and slots[65] == 21 * 64 and slots[134] == 22 * 64 + 5
    assert (slots[135:] == -1).all()


def test_tables_refuse():
    old = np.full((5, 2), 6)
    table, cu, lens, slots, counts = paged.build_tables([0, -1, 0, 64, 0], [64, 3, 129, 64, 1], [0], 4, old, 300)
    # negative | longer than the table | the pages run out, for the last request too
    assert counts.tolist() == [1, 4] and lens.tolist() == [64, 0, 0, 64, 0]
    assert cu.tolist() == [0, 64, 67, 196, 260, 261]
    assert table.tolist() == [[0, -1], [-1, -1], [-1, -1], [6, -1], [-1, -1]]
    assert (slots[:64] >= 0).all() and (slots[64:] == -1).all()


def test_attention_is_one_softmax_over_prefix_and_own():
    """A prefix cached once gives what the same tokens in front of each sequence give."""
    rng = np.random.default_rng(0)
    P, lens, H = 70, [3, 65], 2
    pool = rng.standard_normal((8, 2, H, 64, 64))
    pre, own = [6, 1], np.array([[3, 0], [2, 5]])
    q = rng.standard_normal((2, H, 64))
    out = paged.shared_attention(q, pool, pre, P, own, lens, None)
    for b in range(2):
        at = [(pre[t // 64], t % 64) for t in range(P)] + [(own[b, t // 64], t % 64) for t in range(lens[b])]
        for h in range(H):
            k, v = (np.stack([pool[p, j, h, s] for p, s in at]) for j in (0, 1))
            w = np.exp(k @ q[b, h] / 8)
            np.testing.assert_allclose(out[b, h], (w[:, None] * v).sum(0) / w.sum(), rtol=1e-12)


def test_attention_rows_are_causal_and_empty_rows_are_zero():
    rng = np.random.default_rng(1)
    pool = rng.standard_normal((2, 2, 1, 64, 64))
    q = rng.standard_normal((4, 1, 64))
    a = paged.shared_attention(q, pool, [], 0, np.array([[1]]), [4], [0, 4])
    np.testing.assert_allclose(a[0, 0], pool[1, 1, 0, 0])           # its own token only
    pool[1, :, 0, 3] = 50.0
    b = paged.shared_attention(q, pool, [], 0, np.array([[1]]), [4], [0, 4])
    assert np.array_equal(a[:3], b[:3]) and not np.array_equal(a[3], b[3])
    c = paged.shared_attention(q, pool, [], 0, np.array([[1]]), [2], [0, 4])  # two rows before the first token
    assert (c[:2] == 0).all() and (c[2:] != 0).any()
    assert (paged.shared_attention(q[:1], pool, [0], 5, np.array([[1]]), [-1], None) == 0).all()


# ---- refusals --------------------------------------------------------------------------------
def _tables(B=2, cached=FAKE, added=FAKE + 0x1000, free=FAKE + 0x2000, n_free=4, n_pages=8, table=FAKE + 0x3000, max_pages=3,
            cu=FAKE + 0x4000, lens=FAKE + 0x5000, slots=FAKE + 0x6000, rows=50, counts=FAKE + 0x7000):
    return ftts.lib().ftts_build_tables(cached, added, B, free, n_free, n_pages, table, max_pages, cu, lens, slots, rows,
                                        counts, None)


@pytest.mark.parametrize("bad,code", [
    (dict(added=None), -1), (dict(table=None), -1), (dict(cu=None), -1), (dict(counts=None), -1), (dict(slots=None), -1),
    (dict(free=None), -1), (dict(n_free=-1), -1), (dict(B=0), -2), (dict(B=1025), -2), (dict(max_pages=0), -2),
    (dict(max_pages=513), -2), (dict(n_pages=0), -2), (dict(n_pages=1 << 25), -2), (dict(rows=-1), -5),
    (dict(rows=(1 << 24) + 1), -5), (dict(lens=FAKE), -1), (dict(lens=FAKE + 4), -1), (dict(cu=FAKE + 0x1000 + 4), -1),
    (dict(slots=FAKE + 0x4000), -1), (dict(counts=FAKE + 0x3000 + 20), -1), (dict(table=FAKE + 0x2000), -1),
    (dict(slots=FAKE + 0x6002), -4), (dict(cached=FAKE + 2), -4)])
def test_build_tables_refusals(bad, code):
    assert _tables(**bad) == code, ftts.lib().ftts_last_error()


def _append(src=1, dst=1, k=FAKE, ks=128, v=FAKE + 256, vs=128, rows=3, slots=FAKE, base=FAKE, n_pages=4, layer=0, heads=2):
    kv = ftts.KvPool(base, n_pages)
    return ftts.lib().ftts_append_kv(src, dst, k, ks, v, vs, rows, slots, ctypes.byref(kv), layer, heads, None)


@pytest.mark.parametrize("bad,code", [
    (dict(src=2), -3), (dict(dst=7), -3), (dict(src=1, dst=0), -3), (dict(base=None), -1), (dict(k=None), -1),
    (dict(v=None), -1), (dict(slots=None), -1), (dict(rows=-1), -5), (dict(rows=(1 << 24) + 1), -5), (dict(heads=0), -2),
    (dict(heads=257), -2), (dict(n_pages=0), -2), (dict(layer=-1), -2), (dict(ks=127), -2), (dict(vs=132), -2),
    (dict(ks=120), -2), (dict(src=0, dst=0, ks=130), -2), (dict(k=FAKE + 8), -4), (dict(v=FAKE + 4), -4),
    (dict(base=FAKE + 2), -4), (dict(slots=FAKE + 1), -4)])
def test_append_refusals(bad, code):
    assert _append(**bad) == code, ftts.lib().ftts_last_error()


def test_append_of_no_rows_is_no_call():
    assert _append(rows=0) == 0 and _append(rows=0, k=None, v=None, slots=None) == 0


def _attend(dtype=1, H=4, KH=4, D=64, q=FAKE, qs=256, cu=None, T=2, B=2, prefix=(FAKE, 10), table=FAKE, lens=FAKE,
            max_pages=3, base=FAKE, n_pages=9, layer=0, out=FAKE, os=256, ws=FAKE, ws_bytes=1 << 40):
    s, pt, kv = ftts.AttnShape(dtype, H, KH, D), ftts.PageTable(table, lens, max_pages), ftts.KvPool(base, n_pages)
    p = ctypes.byref(ftts.SharedPrefixC(*prefix)) if prefix else None
    return ftts.lib().ftts_shared_attention(ctypes.byref(s), q, qs, cu, T, B, p, ctypes.byref(pt), ctypes.byref(kv), layer,
                                            out, os, ws, ws_bytes, None)


@pytest.mark.parametrize("bad,code", [
    (dict(dtype=2), -3), (dict(D=128), -7), (dict(H=0), -2), (dict(H=260, qs=260 * 64, os=260 * 64), -2), (dict(KH=0), -2),
    (dict(KH=3), -2), (dict(KH=8), -2), (dict(B=0), -2), (dict(B=65, T=65), -2), (dict(T=3), -2), (dict(T=-1, cu=FAKE), -5),
    (dict(T=(1 << 24) + 1, cu=FAKE), -5), (dict(prefix=(FAKE, -1)), -5), (dict(prefix=(FAKE, (1 << 20) + 1)), -5),
    (dict(prefix=(None, 5)), -1), (dict(table=None), -1), (dict(lens=None), -1), (dict(max_pages=0), -2),
    (dict(max_pages=513), -2), (dict(base=None), -1), (dict(n_pages=0), -2), (dict(layer=-1), -2), (dict(q=None), -1),
    (dict(out=None), -1), (dict(ws=None), -1), (dict(qs=255), -2), (dict(os=260), -2), (dict(qs=248), -2),
    (dict(dtype=0, qs=258), -2), (dict(q=FAKE + 8), -4), (dict(out=FAKE + 2), -4), (dict(base=FAKE + 4), -4),
    (dict(ws=FAKE + 8), -4), (dict(ws_bytes=0), -8)])
def test_shared_attention_refusals(bad, code):
    assert _attend(**bad) == code, ftts.lib().ftts_last_error()


def test_shared_attention_of_no_rows_is_no_call():
    assert _attend(T=0, cu=FAKE, q=None, out=None, ws=None) == 0


def test_workspace_covers_every_smaller_call():
    """Bytes grow with each argument, and arguments that the call refuses give 0."""
    size = ftts.shared_attention_workspace_bytes
    for heads, kv_heads, dtype in ((20, 20, ftts.BF16), (20, 4, ftts.BF16), (1, 1, ftts.F32), (12, 2, ftts.F32)):
        for axis, values in ((0, [1, 3, 16, 64]), (1, [64, 65, 200, 4000, 1 << 18]), (2, [0, 1, 64, 1000, 1 << 20]),
                             (3, [1, 2, 30, 512])):
            at = [64, 64, 1000, 30] if axis else [1, 64, 1000, 30]
            got = []
            for v in values:
                at[axis] = v
                got.append(size(heads, kv_heads, dtype, at[0], at[1], at[2], at[3]))
            assert got == sorted(got) and got[0] > 0, (heads, axis, got)
    for bad in ((20, 3, 1, 1, 1, 1, 1), (20, 20, 3, 1, 1, 1, 1), (20, 20, 1, 65, 65, 1, 1), (20, 20, 1, 1, -1, 1, 1),
                (20, 20, 1, 1, 1, -1, 1), (20, 20, 1, 1, 1, 1, 0)):
        with pytest.raises(ftts.FTTSError):
            size(*bad)


def test_binding_checks():
    """Wrong types and shapes are refused by the binding before any pointer is taken."""
    import torch
    i = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ftts.FTTSError, match="int32"):
        ftts.build_tables(i.long(), i, 4, i.view(2, 1), torch.zeros(3, dtype=torch.int32), i, i)
    with pytest.raises(ftts.FTTSError, match="row_offsets"):
        ftts.build_tables(i, i, 4, i.view(2, 1), i, i, i)
    with pytest.raises(ftts.FTTSError, match="GPU"):
        ftts.build_tables(i, i, 4, i.view(2, 1), torch.zeros(3, dtype=torch.int32), i, i)
    with pytest.raises(ftts.FTTSError, match="hold"):
        ftts.SharedPrefix(i, 129)
    with pytest.raises(ftts.FTTSError, match="pool"):
        ftts.KVCache.over(torch.zeros(1, 2, 2, 1, 32, 64))


# ---- the model behind a shared prefix ----------------------------------------------------------
def test_shared_model_calls_refuse():
    from paper_2607_21042_amd import workload
    from tests.test_abi import _fake_weights
    cfg = ftts.make_config(workload.TINY, ftts.BF16)
    w, L = _fake_weights(cfg), ftts.lib()
    samp, kv = ftts.Sampling(1.0, 1, 1.0), ftts.KvPool(FAKE, 8)

    def step(prefix=(FAKE, 100), B=3, max_pages=4, ws_bytes=1 << 40):
        p = ctypes.byref(ftts.SharedPrefixC(*prefix)) if prefix else None
        pt = ftts.PageTable(FAKE, FAKE, max_pages)
        return L.ftts_decode_step_shared(ctypes.byref(w), p, FAKE, FAKE, ctypes.byref(pt), ctypes.byref(kv), FAKE, None, FAKE,
                                         None, ctypes.byref(samp), B, FAKE, ws_bytes, None)

    def fill(prefix=(FAKE, 100), lens=(3, 4), max_pages=4, ws_bytes=1 << 40):
        p = ctypes.byref(ftts.SharedPrefixC(*prefix)) if prefix else None
        pt, a = ftts.PageTable(FAKE, None, max_pages), (ctypes.c_int32 * len(lens))(*lens)
        z = (ctypes.c_int32 * len(lens))()
        return L.ftts_prefill_shared(ctypes.byref(w), p, FAKE, a, None, z, 0, 0, len(lens), ctypes.byref(pt), ctypes.byref(kv),
                                     FAKE, FAKE, ws_bytes, None)

    for call in (step, fill):
        assert call(prefix=None) == -1 and call(prefix=(None, 3)) == -1
        assert call(prefix=(FAKE, -1)) == -5 and call(prefix=(FAKE, (1 << 20) + 1)) == -5
        assert call(max_pages=0) == -2 and call(ws_bytes=100) == -8
    assert step(B=0) == -2 and step(B=65) == -2 and fill(lens=(0, 4)) == -5 and fill(lens=(257, 4)) == -5
    # a workspace that serves the call without a prefix is too small behind one
    assert step(ws_bytes=ftts.workspace_bytes(cfg, 3, 0)) == -8
    assert fill(ws_bytes=ftts.workspace_bytes(cfg, 2, 7)) == -8
    try:
        ftts.set_decode_path(ftts.PATH_PERSISTENT)
        assert step() == -7 and b"shared prefix" in L.ftts_last_error()
    finally:
        ftts.set_decode_path(ftts.PATH_AUTO)


def test_shared_workspace_covers_smaller_calls():
    from paper_2607_21042_amd import workload
    cfg = ftts.make_config(workload.TINY, ftts.BF16)
    a = ftts.shared_workspace_bytes(cfg, 8, 100, 64, 4)
    assert a > ftts.workspace_bytes(cfg, 8, 100) and a % 256 == 0
    for more in ((16, 100, 64, 4), (8, 4000, 64, 4), (8, 100, 6400, 4), (8, 100, 64, 90)):
        assert ftts.shared_workspace_bytes(cfg, *more) >= a
    for bad in ((0, 1, 1, 1), (65, 1, 1, 1), (1, -1, 1, 1), (1, 1, -1, 1), (1, 1, 1, 0), (1, 1, 1, 513), (1, (1 << 24) + 1, 1, 1)):
        with pytest.raises(ftts.FTTSError):
            ftts.shared_workspace_bytes(cfg, *bad)
