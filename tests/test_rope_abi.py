"""Refusals of the rotary positions' entry points, and their frequencies (CPU: nothing is
launched)."""
import ctypes
import math
import types

import numpy as np
import pytest
import torch

jfkv = pytest.importorskip("paper_2609_17475_amd.jfkv")
L = jfkv.lib
OK, INVALID, UNSUPPORTED = jfkv.JF_OK, jfkv.JF_ERR_INVALID, jfkv.JF_ERR_UNSUPPORTED
ROPE = dict(table=16, rows=None, table_rows=100, rot_dim=64, order=0)
ROTATE = dict(rope=ROPE, dtype=0, d=128, transpose=0, q=16, q_stride=512, q_out=1 << 20,
              q_out_stride=512, hq=4, k=1 << 21, k_stride=128, k_out=1 << 22, k_out_stride=128,
              hk=1, total=3, stream=None)
APPEND = dict(layout=(256, 1, 128, 64, 16), pool=(16, 16, 16, 16), dtype=0, rope=ROPE, k=16,
              k_stride=128, v=16, v_stride=128, q=16, q_stride=512, q_out=1 << 20, hq=4, cu=16,
              start=16, bt=16, B=1, max_pages=4, total=3, stream=None)


def _rope(r):
    if r is None:
        return None
    return ctypes.byref(jfkv.RopeArgs(*dict(ROPE, **r).values()))


def _rotate(**change):
    a = dict(ROTATE, **change)
    return L.jf_rope_rotate(_rope(a.pop("rope")), *a.values())


def _append(**change):
    a = dict(APPEND, **change)
    lay, pool = a.pop("layout"), a.pop("pool")
    a["rope"] = _rope(a["rope"])
    return L.jf_kv8_rope_append(ctypes.byref(jfkv.layout(*lay)) if lay else None,
                                ctypes.byref(jfkv.PoolPtrs(*pool)) if pool else None, *a.values())


@pytest.mark.parametrize("call", [_rotate, _append])
def test_rope_arguments(call):
    for rope, want in ((None, INVALID), (dict(rot_dim=0), INVALID), (dict(rot_dim=-2), INVALID),
                       (dict(rot_dim=63), INVALID), (dict(rot_dim=256), INVALID),
                       (dict(rot_dim=1 << 17), UNSUPPORTED), (dict(order=2), UNSUPPORTED),
                       (dict(order=-1), UNSUPPORTED), (dict(table=None), INVALID),
                       (dict(table=20), INVALID), (dict(rows=18), INVALID),
                       (dict(table_rows=0), INVALID), (dict(table_rows=2), INVALID)):
        assert call(rope=rope) == want, rope
    assert call(dtype=2) == UNSUPPORTED
    assert call(total=-1) == INVALID
    assert call(total=0, q=None, k=None) == OK  # nothing to do


def test_rotate_arguments():
    for change, want in ((dict(d=0), INVALID), (dict(d=127), INVALID), (dict(d=1 << 17), UNSUPPORTED),
                         (dict(hq=-1), INVALID), (dict(hk=-1), INVALID), (dict(q=None), INVALID),
                         (dict(q_out=None), INVALID), (dict(k=None), INVALID),
                         (dict(k_out=None), INVALID), (dict(q=17), INVALID), (dict(k_out=17), INVALID),
                         (dict(q_stride=511), INVALID), (dict(q_stride=-512), INVALID),
                         (dict(k_out_stride=0), INVALID), (dict(k_stride=1 << 40), INVALID),
                         (dict(q_out=16, q_out_stride=520), INVALID),
                         (dict(hq=1 << 20, q_stride=1 << 27, q_out_stride=1 << 27), UNSUPPORTED),
                         (dict(total=1 << 27, rope=dict(table_rows=1 << 27)), UNSUPPORTED)):
        assert _rotate(**change) == want, change
    assert _rotate(hq=0, hk=0, q=None, k=None) == OK


def test_append_arguments():
    for change, want in ((dict(layout=None), INVALID), (dict(layout=(256, 1, 96, 64, 16)), UNSUPPORTED),
                         (dict(pool=None), INVALID), (dict(pool=(16, 16, 24, 16)), INVALID),
                         (dict(rope=dict(rot_dim=40)), UNSUPPORTED), (dict(k=None), INVALID),
                         (dict(v=None), INVALID), (dict(cu=None), INVALID), (dict(start=None), INVALID),
                         (dict(bt=None), INVALID), (dict(q=None), INVALID), (dict(q_out=None), INVALID),
                         (dict(k=24), INVALID), (dict(v=24), INVALID), (dict(q=24), INVALID),
                         (dict(q_out=24), INVALID), (dict(k_stride=127), INVALID),
                         (dict(k_stride=132), INVALID), (dict(v_stride=100), INVALID),
                         (dict(q_stride=504), INVALID), (dict(q_stride=516), INVALID),
                         (dict(q_stride=520, q_out=16), INVALID), (dict(hq=0), INVALID),
                         (dict(B=0), INVALID), (dict(max_pages=0), INVALID),
                         (dict(max_pages=1 << 24), INVALID),
                         (dict(total=(1 << 31) - 1, layout=(256, 1, 128, 16, 4),
                               rope=dict(table_rows=(1 << 31) - 1)), UNSUPPORTED)):
        assert _append(**change) == want, change


def test_table_arguments():
    def call(positions=16, n=4, freq=16, rot=64, magnitude=1.0, table=16):
        return L.jf_rope_table(positions, n, freq, rot, magnitude, table, None)

    for change, want in ((dict(rot=0), INVALID), (dict(rot=5), INVALID), (dict(rot=1 << 17), UNSUPPORTED),
                         (dict(n=-1), INVALID), (dict(magnitude=math.nan), INVALID),
                         (dict(magnitude=math.inf), INVALID), (dict(positions=None), INVALID),
                         (dict(freq=None), INVALID), (dict(table=None), INVALID),
                         (dict(positions=18), INVALID), (dict(freq=18), INVALID),
                         (dict(table=20), INVALID), (dict(n=(1 << 31) - 1), UNSUPPORTED)):
        assert call(**change) == want, change
    assert call(n=0, positions=None) == OK


def _frequencies(rot, base, kind, factor, length, fast, slow):
    """The formulas, in extended precision."""
    x = np.longdouble
    b = x(base) * x(factor) ** (x(rot) / (rot - 2)) if kind == "base" else x(base)
    f = b ** (-2 * np.arange(rot // 2, dtype=x) / rot)
    if kind == "linear":
        return f / factor, 1.0
    if kind != "parts":
        return f, 1.0

    def pair(turns):
        return rot * math.log(length / (2 * math.pi * turns)) / (2 * math.log(base))

    lo, hi = max(math.floor(pair(fast)), 0), min(math.ceil(pair(slow)), rot - 1)
    ramp = np.clip((np.arange(rot // 2, dtype=x) - lo) / x(hi - lo), 0, 1)
    return f * (1 - ramp) + f / x(factor) * ramp, 0.1 * math.log(factor) + 1 if factor > 1 else 1.0


@pytest.mark.parametrize("rot", [4, 16, 64, 128, 256])
@pytest.mark.parametrize("kind,factor", [("plain", 1.0), ("linear", 4.0), ("base", 8.0), ("parts", 8.0),
                                         ("parts", 1.0), ("linear", 0.5)])
def test_frequencies(rot, kind, factor):
    for base, length in ((10000.0, 4096), (500000.0, 8192)):
        got, m = jfkv.rope_frequencies(rot, base, kind, factor, length, 32.0, 1.0)
        want, wm = _frequencies(rot, base, kind, factor, length, 32.0, 1.0)
        assert got.shape == (rot // 2,)
        # one rounding to fp32, after some in 64 bits
        assert np.all(np.abs(got.numpy().astype(np.longdouble) - want) <= want * (2.0 ** -24 + 2.0 ** -45))
        assert abs(m - wm) <= wm * 2.0 ** -24
    if kind == "base":  # what it is for: the fastest pair stays, the slowest is slowed by factor
        assert got[0] == 1.0 and abs(float(got[-1]) * factor * 500000.0 ** (1 - 2 / rot) - 1) < 1e-6


def test_frequency_arguments():
    def call(rot=64, base=1e4, kind=0, factor=2.0, length=4096, fast=32.0, slow=1.0, out=True, mag=True):
        f, m = (ctypes.c_float * 32)(), ctypes.c_float()
        return L.jf_rope_frequencies(rot, base, kind, factor, length, fast, slow,
                                     ctypes.addressof(f) if out else None,
                                     ctypes.addressof(m) if mag else None)

    for change, want in ((dict(rot=0), INVALID), (dict(rot=63), INVALID), (dict(rot=1 << 20), UNSUPPORTED),
                         (dict(kind=4), UNSUPPORTED), (dict(kind=-1), UNSUPPORTED),
                         (dict(out=False), INVALID), (dict(mag=False), INVALID),
                         (dict(base=1.0), INVALID), (dict(base=math.nan), INVALID),
                         (dict(base=math.inf), INVALID), (dict(kind=1, factor=0.0), INVALID),
                         (dict(kind=2, factor=math.nan), INVALID), (dict(kind=2, rot=2), INVALID),
                         (dict(kind=3, length=0), INVALID), (dict(kind=3, slow=0.0), INVALID),
                         (dict(kind=3, fast=1.0), INVALID), (dict(kind=3, fast=math.inf), INVALID)):
        assert call(**change) == want, change
    assert call(factor=-1.0, length=-5, fast=0.0) == OK  # what plain frequencies do not use
    with pytest.raises(ValueError):
        jfkv.rope_frequencies(64, scaling="none")


def test_rows_of_the_binding():
    table = types.SimpleNamespace(table=None, rows=None)  # (looked at after the rows)
    x = torch.zeros(2, 1, 16, dtype=torch.float16)
    for q, q_out in ((None, None), (x, x), (x.float(), x.float())):  # none, on the host, fp32
        with pytest.raises(ValueError):
            jfkv.bind_rope_rotate(table, q, q_out)
