"""How ftts_shared_attention runs a call (ftts_shared_attention_plan, on the host alone): the kernels that the
GPU tests name are the ones that run, every kernel and tile is among their cases, and the workspace holds what
each plan leaves there."""
import random
from types import SimpleNamespace

import numpy as np
import pytest

from paper_2607_21042_amd import ftts
from tests import test_gpu_paged as gpu
from tests import test_gpu_shared_edges as edges

NAMES = {ftts.SHARED_CUT: "cut", ftts.SHARED_WHOLE: "whole", ftts.SHARED_TILE: "tile", ftts.SHARED_PACKED: "packed"}


def plan(dtype, H, KH, B, rows, prompts, prefix, width):
    p = ftts.shared_attention_plan(H, KH, ftts.F32 if dtype == "f32" else ftts.BF16, B, rows, prompts, prefix, width)
    return p, NAMES[p.kernel] + (f" in {p.parts}" if p.parts > 1 else "")


def named(dtype, H, KH, B, rows, prompts, prefix, width):
    """What the GPU tests take a call of these sizes for."""
    return gpu.kernel(SimpleNamespace(f32=dtype == "f32", lens=[1] * B, H=H, KH=KH, P=prefix, width=width,
                                      cu=[0] * (B + 1) if prompts else None, T=rows))


def sizes(rng):
    H, KH = rng.choice([(20, 20), (20, 4), (12, 12), (12, 4), (8, 1), (32, 16), (40, 1), (4, 4), (1, 1), (256, 2)])
    B = rng.choice([1, 2, 3, 8, 31, 32, 33, 64, rng.randint(1, 64)])
    prompts = rng.random() < 0.6
    rows = round(B * 2 ** rng.uniform(0, 10)) + rng.randrange(5) if prompts else B
    prefix = rng.choice([0, 1, 64, 65, round(2 ** rng.uniform(0, 14)), rng.randint(0, 1 << 20)])
    width = rng.choice([1, 2, 5, round(2 ** rng.uniform(0, 9)), 512])
    return rng.choice(["bf16", "bf16", "bf16", "f32"]), H, KH, B, rows, prompts, prefix, width


def test_the_rule_that_the_gpu_tests_restate_is_the_librarys():
    rng, met = random.Random(5), set()
    for _ in range(30000):
        s = sizes(rng)
        got, want = plan(*s)[1], named(*s)
        assert got == want, s
        met.add(got)
    assert met >= {"cut", "whole", "tile", "packed"} | {f"{k} in {n}" for k in ("tile", "packed") for n in (2, 4, 8, 16)}


def test_the_gpu_cases_take_every_kernel():
    for dtype, H, KH, prefix, past, rows, takes in edges.FORMS:
        width = max(-(-(p + n) // 64) for p, n in zip(past, rows or [0] * len(past)))
        assert plan(dtype, H, KH, len(past), sum(rows) if rows else len(past), rows is not None, prefix, width)[1] == takes
    cuts = [plan(d, H, KH, len(past), len(past), False, prefix, max(-(-p // 64) for p in past))[0]
            for d, H, KH, prefix, past, rows, takes in edges.FORMS if takes == "cut" and rows is None]
    # both tiles on both sides
    assert {p.prefix_rows for p in cuts} == {4, 32} and {p.own_rows for p in cuts} == {4, 32}
    for H, KH, prefix, past, rows, takes in [
            (12, 4, 2500, [10, 0, 300], [90, 130, 90], "packed in 8"), (20, 4, 2000, [0, 64, 3, 700], [90, 0, 128, 129], "tile in 4")]:
        width = max(-(-(p + n) // 64) for p, n in zip(past, rows))
        assert plan("bf16", H, KH, len(rows), sum(rows), True, prefix, width)[1] == takes


def test_the_workspace_holds_every_plan():
    """Partial results of 66 floats a row and head; what the host reports is what the launch compares."""
    rng = random.Random(6)
    for _ in range(30000):
        dtype, H, KH, B, rows, prompts, prefix, width = s = sizes(rng)
        p, _ = plan(*s)
        ws = ftts.shared_attention_workspace_bytes(H, KH, ftts.F32 if dtype == "f32" else ftts.BF16, B, rows, prefix, width)
        assert p.partials * rows * H * 66 * 4 <= ws, s
        if p.kernel == ftts.SHARED_CUT:
            runs = [-(-n // c) if n else 0 for n, c in ((-(-prefix // 64), p.prefix_pages), (width, p.own_pages))]
            assert sum(runs) == p.partials and p.parts == 0, s
            assert p.prefix_rows in (4, 32) and p.own_rows in (4, 32)
        else:
            assert (p.prefix_rows, p.own_rows, p.prefix_pages, p.own_pages) == (0, 0, 0, 0)
            assert p.partials == (p.parts if p.parts > 1 else 0)


@pytest.mark.parametrize("args,code", [
    ((20, 3, 1, 1, 1, 0, 1, 1), -2), ((20, 20, 3, 1, 1, 0, 1, 1), -3), ((20, 20, 1, 65, 65, 0, 1, 1), -2),
    ((20, 20, 1, 2, 1, 0, 1, 1), -2), ((20, 20, 1, 2, 0, 1, 1, 1), -2), ((20, 20, 1, 2, -1, 1, 1, 1), -5),
    ((20, 20, 1, 1, 1, 0, -1, 1), -5), ((20, 20, 1, 1, 1, 0, 1, 513), -2)])
def test_plan_refusals(args, code):
    with pytest.raises(ftts.FTTSError) as e:
        ftts.shared_attention_plan(*args)
    assert e.value.code == code
    assert ftts.lib().ftts_shared_attention_plan(None, 1, 1, 0, 0, 1, None) == -1


def test_a_wide_table_takes_longer_runs():
    lens = [np.ceil(n / 64) for n in (700, 65)]
    narrow, wide = (plan("bf16", 20, 20, 32, 32, False, 300, w)[0] for w in (int(max(lens)), 512))
    assert narrow.own_pages < wide.own_pages <= 512
