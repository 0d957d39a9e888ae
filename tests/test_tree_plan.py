"""How ftts_tree_attention runs a call (ftts_tree_attention_plan, on the host alone): every form is among the GPU tests'
cases, a launch stays below 2^32 threads, and the workspace holds its partial results."""
import random

import pytest

from paper_2607_21042_amd import ftts
from tests import test_gpu_tree_forms as gpu

HEADS = [(20, 20), (20, 4), (12, 12), (12, 2), (8, 1), (32, 16), (40, 1), (4, 4), (1, 1), (256, 2), (256, 256)]


def test_the_gpu_cases_take_every_form():
    met = set()
    for dtype, H, KH, past, rows, prefix, width, takes in gpu.FORMS:
        assert len(past) == len(rows) and max(-(-(p + n) // 64) for p, n in zip(past, rows)) <= width
        assert gpu.taken(dtype, H, KH, past, rows, prefix, width) == takes
        met.add((dtype, takes[0], takes[1] > 1, takes[2] > gpu.LISTED))
    every = {(d, w, many, False) for d in ("bf16", "f32") for w in (4, 8) for many in (False, True)}
    forms = {(d, w, many) for d, w, many, _ in met}
    assert forms == {f[:3] for f in every}
    # waves that list their half pages more than once: everywhere but in bf16 with 8 waves and parts, whose parts are short
    assert {f[:3] for f in met if f[3]} == forms - {("bf16", 8, True)}


def test_some_calls_go_in_blocks_and_some_do_not():
    blocks = {ftts.tree_attention_plan(20, 20, ftts.BF16, B, 12 * B, 0, 8).blocks for B in (1, 2, 16, 32)}
    assert blocks == {0, 1}


def test_launches_and_workspaces():
    rng = random.Random(4)
    for _ in range(20000):
        H, KH = rng.choice(HEADS)
        dtype, B, width = rng.choice([ftts.F32, ftts.BF16]), rng.randint(1, 64), rng.choice([1, 2, 9, round(2 ** rng.uniform(0, 9)), 512])
        prefix = rng.choice([0, 1, 65, round(2 ** rng.uniform(0, 20))])
        rows = min(round(2 ** rng.uniform(0, 24.1)), 1 << 24)
        try:
            p = ftts.tree_attention_plan(H, KH, dtype, B, rows, prefix, width)
        except ftts.FTTSError as e:
            assert e.code == -5 and rows * H > (1 << 29) - (1 << 20)
            continue
        assert p.waves in (4, 8) and 1 <= p.parts <= 48 and p.tiles >= rows * (H // KH) // 32 + B
        assert p.tiles * KH * p.parts * p.waves * 64 < 1 << 32
        assert p.parts == 1 or not p.blocks and p.tiles * KH * p.parts % 8 in (0, p.tiles * KH % 8) and KH * p.parts % 8 == 0
        assert not p.blocks or p.tiles % 8 == 0
        partials = p.parts * rows * H if p.parts > 1 else 0
        assert partials * 66 * 4 <= ftts.tree_attention_workspace_bytes(H, KH, dtype, B, rows, prefix, width)


@pytest.mark.parametrize("args,code", [
    ((20, 3, 1, 1, 1, 0, 1), -2), ((20, 20, 3, 1, 1, 0, 1), -3), ((20, 20, 1, 65, 65, 0, 1), -2), ((20, 20, 1, 2, 0, 0, 1), -2),
    ((20, 20, 1, 2, -1, 0, 1), -5), ((20, 20, 1, 1, 1, -1, 1), -5), ((20, 20, 1, 1, 1, 0, 513), -2), ((256, 1, 1, 1, 1 << 22, 0, 1), -5)])
def test_plan_refusals(args, code):
    with pytest.raises(ftts.FTTSError) as e:
        ftts.tree_attention_plan(*args)
    assert e.value.code == code
    assert ftts.lib().ftts_tree_attention_plan(None, 1, 1, 0, 1, None) == -1
