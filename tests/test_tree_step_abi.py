"""Refusals of the model's pass over drafted trees, without a GPU (every call fails before anything is enqueued)."""
import ctypes
from types import SimpleNamespace

import pytest
import torch

from paper_2607_21042_amd import ftts, workload
from tests.test_abi import _fake_weights

FAKE = 0x100000
SHAPE, L = workload.TINY, ftts.lib()
CFG = ftts.make_config(SHAPE, ftts.BF16)
W = _fake_weights(CFG)


def step(w=W, prefix=None, tokens=FAKE, positions=FAKE, cu=FAKE, rows=9, B=2, masks=FAKE, words=1, width=4, lens=FAKE, table=FAKE,
         base=FAKE, pages=8, out=FAKE, ws=FAKE, size=1 << 40):
    pt, kv = ftts.PageTable(table, lens, width), ftts.KvPool(base, pages)
    return L.ftts_tree_step(ctypes.byref(w) if w else None, ctypes.byref(prefix) if prefix else None, tokens, positions, cu, rows, B, masks,
                            words, ctypes.byref(pt), ctypes.byref(kv), out, ws, size, None)


@pytest.mark.parametrize("bad,code", [
    (dict(w=None), -1), (dict(tokens=None), -1), (dict(positions=None), -1), (dict(cu=None), -1), (dict(masks=None), -1),
    (dict(out=None), -1), (dict(table=None), -1), (dict(lens=None), -1), (dict(base=None), -1), (dict(base=FAKE + 8), -4),
    (dict(masks=FAKE + 4), -4), (dict(ws=None), -1), (dict(ws=FAKE + 8), -4), (dict(size=1000), -8), (dict(B=0), -2), (dict(B=65), -2),
    (dict(rows=0), -5), (dict(rows=(1 << 20) + 1), -5), (dict(words=0), -2), (dict(words=5), -2), (dict(width=0), -2),
    (dict(width=513), -2), (dict(pages=0), -2), (dict(prefix=ftts.SharedPrefixC(None, 4)), -1),
    (dict(prefix=ftts.SharedPrefixC(FAKE, -1)), -5), (dict(prefix=ftts.SharedPrefixC(FAKE, (1 << 20) + 1)), -5)])
def test_refused(bad, code):
    assert step(**bad) == code, L.ftts_last_error()


def test_a_workspace_of_another_call_is_too_small():
    need = ftts.tree_workspace_bytes(CFG, 2, 200)
    assert need > ftts.workspace_bytes(CFG, 2, 200) and step(rows=200, size=ftts.workspace_bytes(CFG, 2, 0)) == -8


@pytest.mark.parametrize("wdtype", [ftts.F32, ftts.BF16, ftts.W8A16, ftts.W4A16])
def test_workspaces_cover_smaller_calls(wdtype):
    for shape in (workload.TINY, workload.INDEXTTS2):
        cfg, last = ftts.make_config(shape, wdtype), 0
        for rows in (1, 7, 8, 32, 33, 100, 255, 256, 1000, 5000):
            n = ftts.tree_workspace_bytes(cfg, 16, rows)
            assert n >= last and n >= ftts.workspace_bytes(cfg, 16, rows) and ftts.tree_workspace_bytes(cfg, 1, rows) <= n
            last = n
    for bad in ((0, 5), (65, 5), (4, 0), (4, -1), (4, (1 << 20) + 1)):
        with pytest.raises(ftts.FTTSError):
            ftts.tree_workspace_bytes(cfg, *bad)


def bound(T=9, B=2, tokens=9, positions=9, masks=(9, 1), logits=None, tdtype=torch.int32, mdtype=torch.int64, table=2):
    i = lambda n, t=torch.int32: torch.zeros(n, dtype=t)  # noqa: E731
    pt = SimpleNamespace(block_table=i((table, 2)), seq_lens=i(table), c=ftts.PageTable())
    ftts.tree_step(SimpleNamespace(shape=SHAPE, wdtype=ftts.BF16, c=ftts.Weights()), i(tokens, tdtype), i(positions), i(B + 1),
                   i(masks, mdtype), pt, SimpleNamespace(pool=torch.zeros(1), c=ftts.KvPool()), torch.zeros(T * SHAPE.vocab if logits is None else logits),
                   torch.zeros(16, dtype=torch.uint8))


@pytest.mark.parametrize("bad,what", [
    (dict(tdtype=torch.int64), "tokens"), (dict(positions=8), "positions"), (dict(masks=(8, 1)), "masks"), (dict(masks=(9,)), "masks"),
    (dict(mdtype=torch.int32), "masks"), (dict(logits=9 * SHAPE.vocab - 1), "logits_out"), (dict(table=1), "page table"),
    (dict(), "GPU")])
def test_binding_refuses_before_the_library(bad, what):
    with pytest.raises(ftts.FTTSError, match=what):
        bound(**bad)


def test_binding_refuses_a_prefix_on_another_device():
    def call(length):
        pages = SimpleNamespace(get_device=lambda: 1)
        i = lambda *n: torch.zeros(n, dtype=torch.int32)  # noqa: E731
        ftts.tree_step(SimpleNamespace(shape=SHAPE, wdtype=ftts.BF16, c=ftts.Weights()), i(9), i(9), i(3), torch.zeros((9, 1), dtype=torch.int64),
                       SimpleNamespace(block_table=i(2, 2), seq_lens=i(2), c=ftts.PageTable()), SimpleNamespace(pool=torch.zeros(1), c=ftts.KvPool()),
                       torch.zeros(9 * SHAPE.vocab), torch.zeros(16, dtype=torch.uint8),
                       prefix=SimpleNamespace(pages=pages, len=length, c=ftts.SharedPrefixC()))
    with pytest.raises(ftts.FTTSError, match="prefix must be on"):
        call(5)
    with pytest.raises(ftts.FTTSError, match="GPU"):        # (a prefix of no tokens has no pages to read)
        call(0)
