"""Refusals of the attention of requests that share prefixes (CPU: nothing is launched)."""
import ctypes
import math

import pytest

jfkv = pytest.importorskip("paper_2609_17475_amd.jfkv")
L = jfkv.lib
OK, INVALID, UNSUPPORTED = jfkv.JF_OK, jfkv.JF_ERR_INVALID, jfkv.JF_ERR_UNSUPPORTED
CALL = dict(layout=(256, 8, 128, 64, 16), pool=(16, 16, 16, 16), dtype=0, q=16, B=4, sq=1, hq=32, bt=16,
            max_pages=4, lens=16, first=16, shared=16, groups=2, scale=1.0, ws=16, ws_bytes=1 << 40,
            out=16, lse=None, stream=None)


def _call(**change):
    a = dict(CALL, **change)
    lay, pool = a.pop("layout"), a.pop("pool")
    return L.jf_kv8_shared_attn(ctypes.byref(jfkv.layout(*lay)) if lay else None,
                                ctypes.byref(jfkv.PoolPtrs(*pool)) if pool else None, *a.values())


@pytest.mark.parametrize("change,want", [
    (dict(layout=None), INVALID), (dict(layout=(256, 0, 128, 64, 4)), INVALID),
    (dict(layout=(256, 8, 96, 64, 4)), UNSUPPORTED), (dict(layout=(100, 8, 128, 64, 4)), UNSUPPORTED),
    (dict(layout=(256, 8, 128, 48, 4)), UNSUPPORTED), (dict(pool=None), INVALID),
    (dict(pool=(16, None, 16, 16)), INVALID), (dict(pool=(16, 16, 24, 16)), INVALID),
    (dict(dtype=2), UNSUPPORTED), (dict(B=0), INVALID), (dict(B=-1), INVALID),
    (dict(B=70000, hq=8), UNSUPPORTED), (dict(B=4000), UNSUPPORTED), (dict(sq=0), UNSUPPORTED),
    (dict(sq=5), UNSUPPORTED), (dict(hq=0), INVALID), (dict(hq=12), INVALID), (dict(max_pages=0), INVALID),
    (dict(max_pages=1 << 23), INVALID), (dict(groups=0), INVALID), (dict(groups=-1), INVALID),
    (dict(groups=5), INVALID), (dict(scale=math.nan), INVALID), (dict(scale=math.inf), INVALID),
    (dict(scale=2.0 ** 126), INVALID), (dict(q=None), INVALID), (dict(bt=None), INVALID),
    (dict(lens=None), INVALID), (dict(first=None), INVALID), (dict(shared=None), INVALID),
    (dict(ws=None), INVALID), (dict(out=None), INVALID), (dict(q=24), INVALID), (dict(out=24), INVALID),
    (dict(ws=24), INVALID), (dict(lse=18), INVALID), (dict(ws_bytes=1000), INVALID)])
def test_refusals(change, want):
    assert _call(**change) == want


def test_workspace_bytes():
    def need(B=4, G=2, sq=1, hq=32, lay=(256, 8, 128, 64, 16)):
        return jfkv.jf_kv8_shared_workspace_bytes(jfkv.layout(*lay), B, G, sq, hq)

    # does not depend on the pool or on lengths, grows with the batch
    assert need() == need(lay=(256, 8, 128, 64, 1000)) == need(lay=(64, 8, 128, 16, 16))
    assert need() <= need(B=8) <= need(B=8, sq=4)
    lay = jfkv.layout(256, 8, 128, 64, 16)
    assert L.jf_kv8_shared_workspace_bytes(ctypes.byref(lay), 4, 2, 1, 32, None) == INVALID
    for change, want in ((dict(B=0), INVALID), (dict(G=0), INVALID), (dict(G=5), INVALID),
                         (dict(hq=30), INVALID), (dict(sq=5), UNSUPPORTED), (dict(B=2049), UNSUPPORTED)):
        with pytest.raises(jfkv.JfError) as e:
            need(**change)
        assert e.value.status == want
