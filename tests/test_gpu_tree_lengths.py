"""Lengths at the ends of their type behind drafted trees: one below a sequence's rows makes it inactive down to -2^31, one
past the table ends there up to 2^31 - 1."""
import numpy as np
import pytest

from tests import test_gpu_tree_step as step
from tests.test_gpu_commit import Drafts, chain_plan, random_plan
from tests.test_gpu_tree import Trees

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
LEAST = -2 ** 31


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_commit_keeps_nothing_of_the_least_lengths(dtype):
    rows = [5, 9, 3, 256, 1, 40, 2]
    d = Drafts(dtype, 2, 3, [60, 0, 20, 5, 9, 70, 30], rows, chain_plan(2, 9), 8)
    for b, n in ((1, LEAST), (2, LEAST + 2), (3, LEAST + 255), (4, LEAST), (5, LEAST + 40)):
        d.lens[b] = n
    print(f"commit: {dtype}, lengths {d.lens}", flush=True)
    d.gpu().call()
    want = d.check()
    assert want[1].tolist() == [3, 0, 0, 0, 0, 0, 1] and want[3].tolist()[1:6] == d.lens[1:6]
    d = Drafts(dtype, 1, 1, [3] * 64, [7] * 64, random_plan(2, 4), 6)
    d.lens = [LEAST + b for b in range(64)]
    d.gpu().call()
    assert not d.check()[1].any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("every", [1, 2, 29])
def test_commit_behind_the_largest_lengths(dtype, every):
    """Paths whose places lie past every table move nothing; counts and new lengths are a path's as elsewhere."""
    rows = [3, 9, 256, 30, 200]
    d = Drafts(dtype, 2, 3, [60, 0, 20, 5, 9], rows, chain_plan(every, 999), 200, width=5)
    for b, n in ((0, 2 ** 31 - 1), (1, 2 ** 31 - 1), (2, 2 ** 31 - 1), (3, 2 ** 31 - 9)):
        d.lens[b] = n
    print(f"commit: {dtype}, every {every}, lengths {d.lens}", flush=True)
    d.gpu().call()
    want = d.check()
    assert want[1].tolist() == [min(-(-n // every), 200) for n in rows]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("prefix", [0, 70])
def test_attention_of_the_least_and_the_largest_lengths(dtype, prefix):
    """Rows of a sequence whose length is from -2^31 on are 0; a length past the table sees what the table holds."""
    rows = [3, 9, 100, 40, 2, 5, 70]
    t = Trees(dtype, 4, 2, prefix, [100, 0, 5, 60, 141, 123, 58], rows, width=2)
    for b, n in ((1, LEAST), (2, LEAST + 99), (3, LEAST + 39), (4, LEAST), (5, 2 ** 31 - 1), (6, 2 ** 31 - 3)):
        t.lens[b] = n
    print(f"attention: {dtype}, prefix {prefix}, lengths {t.lens}", flush=True)
    t.gpu().call()
    few = [min(n, 2 * 64 + r) for n, r in zip(t.lens, rows)]       # (the oracle lists a sequence's tokens)
    t.lens = few
    t.check()
    assert (t.out[t.cu[1]:t.cu[5]] == 0).all() and (t.out[t.cu[5]:t.cu[7]] != 0).any(1).all()


@pytest.mark.parametrize("mode", ["f32", "bf16"])
def test_tree_step_of_the_least_lengths(mode):
    """A sequence whose length is from -2^31 on writes no key and value, and the others' logits are as beside any inactive
    one."""
    dm = step.ftts.DeviceModel(step.weights(mode), step.SHAPE, step.MODES[mode])
    rng = np.random.default_rng(6)
    trees = [step.random_tree(rng, n) for n in (5, 9, 3)]
    r = step.Run(dm, mode, [30, 4, 61], 40)
    clean = r.kv.pool.clone()
    want = r.step([30, -7, 61], trees, [0, 0, 0])
    after = r.kv.pool.clone()
    assert not torch.equal(after.nan_to_num(), clean.nan_to_num())
    for length in (LEAST, LEAST + 8):
        r.kv.pool.copy_(clean)
        got = r.step([30, length - 9, 61], trees, [0, 0, 0])
        assert np.array_equal(got[:5], want[:5]) and np.array_equal(got[14:], want[14:])
        assert torch.equal(r.kv.pool.nan_to_num(), after.nan_to_num())
