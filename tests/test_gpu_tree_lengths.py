"""Lengths at the ends of their type behind drafted trees: one below a sequence's rows makes it inactive down to -2^31, one
past the table ends there up to 2^31 - 1."""
import numpy as np
import pytest

from tests.test_gpu_commit import Drafts, chain_plan, random_plan

pytestmark = pytest.mark.gpu
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
@pytest.mark.parametrize("step", [1, 2, 29])
def test_commit_behind_the_largest_lengths(dtype, step):
    """Paths whose places lie past every table move nothing; counts and new lengths are a path's as elsewhere."""
    rows = [3, 9, 256, 30, 200]
    d = Drafts(dtype, 2, 3, [60, 0, 20, 5, 9], rows, chain_plan(step, 999), 200, width=5)
    for b, n in ((0, 2 ** 31 - 1), (1, 2 ** 31 - 1), (2, 2 ** 31 - 1), (3, 2 ** 31 - 9)):
        d.lens[b] = n
    print(f"commit: {dtype}, step {step}, lengths {d.lens}", flush=True)
    d.gpu().call()
    want = d.check()
    assert want[1].tolist() == [min(-(-n // step), 200) for n in rows]
