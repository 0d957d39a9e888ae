"""Tensors that do not fit the batch are refused by the binding of the model calls behind a shared prefix, and
by the scheduler, before any pointer is taken (no GPU)."""
from types import SimpleNamespace

import numpy as np
import pytest
import torch

from paper_2607_21042_amd import ftts, serve, workload

SHAPE, D, V = workload.TINY, workload.TINY.d_model, workload.TINY.vocab
I, F, H = torch.int32, torch.float32, torch.bfloat16


def table(B):
    return SimpleNamespace(block_table=torch.zeros((B, 2), dtype=I), seq_lens=torch.zeros(B, dtype=I), c=ftts.PageTable())


def model():
    return SimpleNamespace(shape=SHAPE, wdtype=ftts.BF16, c=ftts.Weights())


PREFIX, KV, WS = SimpleNamespace(c=ftts.SharedPrefixC()), SimpleNamespace(c=ftts.KvPool()), torch.zeros(16, dtype=torch.uint8)


def fill(emb=(5, D), dtype=H, cond=(2, 3), ids=4, text=(1, 3), B=2, logits=2 * V):
    ftts.prefill_shared(model(), PREFIX, None if emb is None else torch.zeros(emb, dtype=dtype), cond,
                        torch.zeros(ids, dtype=I), text, 10, 0, table(B), KV, torch.zeros(logits), WS)


@pytest.mark.parametrize("bad,what", [
    (dict(text=(1,)), "text_lens"), (dict(text=(1, 3, 0)), "text_lens"), (dict(emb=(5, D - 1)), "cond_emb"),
    (dict(emb=(4, D)), "cond_emb"), (dict(dtype=F), "cond_emb"), (dict(emb=None), "cond_emb"), (dict(ids=3), "text_ids"),
    (dict(B=1), "page table"), (dict(logits=2 * V - 1), "last_logits")])
def test_prefill_shared_refuses(bad, what):
    with pytest.raises(ftts.FTTSError, match=what):
        fill(**bad)


def step(tokens=3, positions=3, B=3, logits=(3, V), out=3, uniforms=3, hidden=(3, D), tdtype=I):
    ftts.decode_step_shared(model(), PREFIX, torch.zeros(tokens, dtype=tdtype), torch.zeros(positions, dtype=I), table(B), KV,
                            torch.zeros(logits), torch.zeros(out, dtype=I), torch.zeros(uniforms), ftts.Sampling(1.0, 1, 1.0), WS,
                            hidden_out=torch.zeros(hidden))


@pytest.mark.parametrize("bad,what", [
    (dict(tdtype=torch.int64), "tokens"), (dict(positions=2), "positions"), (dict(B=2), "page table"),
    (dict(logits=(3, V - 1)), "logits_out"), (dict(out=2), "sampled_out"), (dict(uniforms=2), "uniforms"),
    (dict(hidden=(2, D)), "hidden_out")])
def test_decode_step_shared_refuses(bad, what):
    with pytest.raises(ftts.FTTSError, match=what):
        step(**bad)


def test_what_fits_goes_on_to_the_pointers():
    for call in (fill, step, lambda: fill(B=5), lambda: step(B=4)):
        with pytest.raises(ftts.FTTSError, match="GPU"):
            call()


def test_the_scheduler_refuses_rows_of_another_width():
    with pytest.raises(ValueError, match="shared_prefix"):
        serve.Scheduler(model(), SHAPE, 1, 8, 64, None, graphs=False, shared_prefix=np.zeros((3, D + 1), dtype=np.float32))
    with pytest.raises(ValueError, match="shared_prefix"):
        serve.Scheduler(model(), SHAPE, 1, 8, 64, None, graphs=False, shared_prefix=np.zeros(D, dtype=np.float32))
    s = serve.Scheduler.__new__(serve.Scheduler)
    s.shape, s.max_pages, s.pool, s.slot_pages, s.waiting, s.next_rid = SHAPE, 3, ftts.PagePool(4), [[]], [], 0
    with pytest.raises(ValueError, match="d_model"):
        s.submit(serve.Request(prefix=np.zeros((3, D - 1), dtype=np.float32), max_new=2))
    s.submit(serve.Request(prefix=np.zeros((3, D), dtype=np.float32), max_new=2))
