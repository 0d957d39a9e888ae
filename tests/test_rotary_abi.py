"""Refusals of the rotation's entry points, and the frequencies that ftts_rotary_init makes, without a GPU (every call
below fails before anything is enqueued)."""
import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import tree
from paper_2607_21042_amd import ftts

FAKE = 0x100000
L = ftts.lib()


@pytest.mark.parametrize("dim", [2, 4, 20, 64])
@pytest.mark.parametrize("scaling", [ftts.ROTARY_PLAIN, ftts.ROTARY_LINEAR, ftts.ROTARY_BASE, ftts.ROTARY_PARTS])
def test_frequencies(dim, scaling):
    if scaling == ftts.ROTARY_BASE and dim == 2:
        pytest.skip("a larger base needs two pairs")
    r = ftts.Rotary(dim, ftts.ROTARY_PAIRS, 500000.0, scaling, 8.0, 4096, 1.0, 4.0)
    f, scale = tree.frequencies(dim, 500000.0, scaling, 8.0, 4096.0, 1.0, 4.0)
    assert len(r.turns) == dim // 2
    # a power and a division in fp64: a few steps of 2^-53
    assert np.allclose(r.turns, f / (2 * math.pi), rtol=2 ** -49, atol=0) and r.c.scale == np.float32(scale)
    assert ftts.Rotary(64, scale=0.5).c.scale == 0.5


@pytest.mark.parametrize("bad,code", [
    (dict(dim=0), -2), (dict(dim=66), -2), (dict(dim=7), -2), (dict(layout=2), -1), (dict(base=1.0), -5),
    (dict(base=math.inf), -5), (dict(base=math.nan), -5), (dict(scaling=4), -1), (dict(scaling=-1), -1),
    (dict(scaling=1, factor=0.5), -5), (dict(scaling=2, factor=math.nan), -5), (dict(scaling=2, dim=2, factor=2.0), -2),
    (dict(scaling=2, base=1e300, dim=4, factor=1e300), -5), (dict(scaling=3, factor=2.0, original=0), -5),
    (dict(scaling=3, factor=2.0, slow=4.0, fast=4.0), -5), (dict(scaling=3, factor=2.0, slow=-1.0), -5)])
def test_frequencies_refused(bad, code):
    with pytest.raises(ftts.FTTSError) as e:
        ftts.Rotary(**bad)
    assert e.value.code == code


def turn(**change):
    r = ftts.RotaryC()
    assert L.ftts_rotary_init(64, 0, 10000.0, 0, 1.0, 1.0, 1.0, 2.0, ctypes.byref(r)) == 0
    r.dim, r.layout, r.scale = change.get("dim", 64), change.get("layout", 0), change.get("scale", 1.0)
    r.turns[5] = change.get("turns", 0.1)
    return r


def rotate(src=1, dst=1, rot=None, x=FAKE, xs=1280, rows=4, heads=20, pos=FAKE, out=FAKE * 4, outs=1280):
    return L.ftts_rotate(src, dst, None if rot == 0 else ctypes.byref(rot or turn()), x, xs, rows, heads, pos, out, outs, None)


@pytest.mark.parametrize("bad,code", [
    (dict(src=2), -3), (dict(dst=7), -3), (dict(src=1, dst=0), -3), (dict(rot=0), -1), (dict(rot=turn(dim=63)), -2),
    (dict(rot=turn(dim=66)), -2), (dict(rot=turn(layout=3)), -1), (dict(rot=turn(scale=math.inf)), -5),
    (dict(rot=turn(turns=1.5)), -5), (dict(rot=turn(turns=math.nan)), -5), (dict(rows=-1), -5), (dict(rows=(1 << 24) + 1), -5),
    (dict(heads=0), -2), (dict(heads=257), -2), (dict(x=None), -1), (dict(out=None), -1), (dict(pos=None), -1), (dict(pos=FAKE + 2), -4),
    (dict(xs=1272 + 4), -2), (dict(xs=1216), -2), (dict(outs=1284), -2), (dict(x=FAKE + 8), -4), (dict(out=FAKE * 4 + 2), -4),
    (dict(out=FAKE + 2560), -1), (dict(out=FAKE - 128), -1), (dict(src=0, out=FAKE), -1),
    (dict(xs=2560, outs=2560, out=FAKE + 1280), -1), (dict(xs=1280, outs=2560, out=FAKE), -1)])
def test_rotate_refused(bad, code):
    assert rotate(**bad) == code, L.ftts_last_error()
    assert b"rotate" in L.ftts_last_error()


def append(src=1, dst=1, rot=None, q=FAKE, qs=3840, heads=20, qo=FAKE * 16, qos=1280, k=FAKE + 2560, ks=3840, v=FAKE + 5120, vs=3840,
           rows=4, pos=FAKE, slots=FAKE, base=FAKE * 64, pages=4, layer=0, kvh=20):
    kv = ftts.KvPool(base, pages)
    return L.ftts_append_rotated(src, dst, ctypes.byref(rot or turn()), q, qs, heads, qo, qos, k, ks, v, vs, rows, pos, slots,
                                 ctypes.byref(kv), layer, kvh, None)


@pytest.mark.parametrize("bad,code", [
    (dict(src=3), -3), (dict(src=1, dst=0), -3), (dict(rot=turn(dim=1)), -2), (dict(base=None), -1), (dict(base=FAKE + 8), -4),
    (dict(heads=-1), -2), (dict(heads=257), -2), (dict(kvh=0), -2), (dict(kvh=257), -2), (dict(pages=0), -2), (dict(layer=-1), -2),
    (dict(heads=0), -2), (dict(heads=0, q=None), -2), (dict(q=None), -1), (dict(qo=None), -1), (dict(k=None), -1), (dict(v=None), -1),
    (dict(pos=None), -1), (dict(slots=None), -1), (dict(slots=FAKE + 1), -4), (dict(ks=1200), -2), (dict(vs=3844), -2),
    (dict(k=FAKE + 2564), -4), (dict(rows=-2), -5), (dict(qo=FAKE + 128, qos=3840), -1), (dict(qo=FAKE + 2560, qos=3840), -1),
    (dict(qo=FAKE + 5120, qos=3840), -1), (dict(src=0, qo=FAKE, qos=7680), -1)])
def test_append_refused(bad, code):
    assert append(**bad) == code, L.ftts_last_error()


def test_nothing_to_do_is_fine():
    assert rotate(rows=0) == 0 and rotate(rows=0, x=None, out=None, pos=None) == 0
    assert append(rows=0) == 0 and append(rows=0, heads=0, q=None, qo=None, k=None, v=None) == 0


def test_binding_refuses_before_the_library():
    x, pos = torch.zeros((3, 128), dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int32)
    r, kv = ftts.Rotary(), type("kv", (), {"pool": torch.zeros((1, 2, 2, 2, 64, 64), dtype=torch.bfloat16), "dtype": ftts.BF16, "c": ftts.KvPool()})
    for call, code in ((lambda: ftts.rotate(x[:, :100], r, pos, x), -2), (lambda: ftts.rotate(x.half(), r, pos, x), -3),
                       (lambda: ftts.rotate(x, r, pos.long(), x), -3), (lambda: ftts.rotate(x, r, pos[:2], x), -2),
                       (lambda: ftts.rotate(x, r, pos, x[:2]), -2), (lambda: ftts.rotate(x, r, pos, x), -1),
                       (lambda: ftts.append_rotated(x, x, r, pos, pos, kv, 1), -5), (lambda: ftts.append_rotated(x, x, r, pos, pos, kv, 0, q=x), -1),
                       (lambda: ftts.append_rotated(x, x.float(), r, pos, pos, kv, 0), -3),
                       (lambda: ftts.append_rotated(x, x, r, pos, pos, kv, 0, q=x, q_out=x.float()), -3),
                       (lambda: ftts.append_rotated(x[:, :64], x, r, pos, pos, kv, 0), -2), (lambda: ftts.append_rotated(x, x, r, pos, pos, kv, 0), -1)):
        with pytest.raises(ftts.FTTSError) as e:
            call()
        assert e.value.code == code, e.value
