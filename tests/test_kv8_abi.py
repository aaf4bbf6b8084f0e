"""Refusals of the 8-bit cache's entry points (CPU: nothing is launched)."""
import ctypes

import pytest

jfkv = pytest.importorskip("paper_2609_17475_amd.jfkv")
L = jfkv.lib
OK, INVALID, UNSUPPORTED = jfkv.JF_OK, jfkv.JF_ERR_INVALID, jfkv.JF_ERR_UNSUPPORTED
LAY = (256, 8, 128, 64, 16)
BIG = 1 << 40
NAN, INF = float("nan"), float("inf")


def _call(fn, spec, change):
    """fn with the arguments of spec (name, value), some of them changed."""
    args = dict(spec)
    assert set(change) <= set(args), change
    args.update(change)
    lay = args.pop("layout")
    ptrs = args.pop("pool", None)
    lay = None if lay is None else ctypes.byref(jfkv.layout(*lay))
    head = [lay] if "pool" not in dict(spec) else \
        [lay, None if ptrs is None else ctypes.byref(jfkv.PoolPtrs(*ptrs))]
    return fn(*head, *args.values())


POOL = (16, 16, 16, 16)
APPEND = [("layout", LAY), ("pool", POOL), ("dtype", 0), ("k", 16), ("v", 16), ("cu", 16),
          ("start", 16), ("bt", 16), ("B", 1), ("max_pages", 4), ("total", 1), ("stream", None)]
DECODE = [("layout", LAY), ("pool", POOL), ("dtype", 0), ("q", 16), ("B", 1), ("sq", 1), ("hq", 32),
          ("bt", 16), ("max_pages", 4), ("lens", 16), ("scale", 1.0), ("splits", 8), ("ws", 16),
          ("ws_bytes", BIG), ("out", 16), ("weights", None), ("stride", 0), ("stream", None)]
PREFILL = [("layout", LAY), ("pool", POOL), ("dtype", 0), ("q", 16), ("T", 16), ("hq", 32),
           ("bt", 16), ("max_pages", 4), ("prefix", 10), ("scale", 1.0), ("ws", 16),
           ("ws_bytes", BIG), ("out", 16), ("lse", 16), ("stream", None)]
WEIGHTS = [("layout", LAY), ("pool", POOL), ("dtype", 0), ("q", 16), ("lse", 16), ("T", 16),
           ("hq", 32), ("bt", 16), ("max_pages", 4), ("prefix", 10), ("scale", 1.0), ("w", 16),
           ("stride", 1024), ("stream", None)]
EVICT = [("layout", LAY), ("pool", POOL), ("B", 1), ("bt", 16), ("max_pages", 4), ("lens", 16),
         ("w", 16), ("stride", 1024), ("keep", 100), ("recent", 10), ("dst", 16), ("dst_pages", 1),
         ("ws", 16), ("ws_bytes", BIG), ("kept", 16), ("kept_w", 16), ("stream", None)]
CALLS = [(L.jf_kv8_append, APPEND), (L.jf_kv8_decode_attn, DECODE), (L.jf_kv8_prefill_attn, PREFILL),
         (L.jf_kv8_attn_weights, WEIGHTS), (L.jf_kv8_evict, EVICT)]


@pytest.mark.parametrize("fn,spec", CALLS, ids=lambda x: getattr(x, "__name__", ""))
def test_layouts_and_pools(fn, spec):
    for lay, want in ((None, INVALID), ((256, 0, 128, 64, 4), INVALID), ((256, 8, 128, 0, 4), INVALID),
                      ((256, 8, 128, 64, -1), INVALID), ((256, 8, 96, 64, 4), UNSUPPORTED),
                      ((256, 8, 128, 48, 4), UNSUPPORTED), ((256, 8, 128, 8, 4), UNSUPPORTED),
                      ((256, 8, 128, 256, 4), UNSUPPORTED), ((100, 8, 128, 64, 4), UNSUPPORTED),
                      ((64, 8, 128, 128, 4), UNSUPPORTED), ((8192, 8, 128, 64, 4), UNSUPPORTED),
                      ((256, 1 << 12, 128, 64, 1 << 20), UNSUPPORTED)):
        assert _call(fn, spec, {"layout": lay}) == want, lay
    assert _call(fn, spec, {"pool": None}) == INVALID
    for i in range(4):
        p = list(POOL)
        p[i] = None
        assert _call(fn, spec, {"pool": tuple(p)}) == INVALID
    assert _call(fn, spec, {"pool": (24, 16, 16, 16)}) == INVALID
    assert b"aligned" in L.jf_last_error()


@pytest.mark.parametrize("fn,spec", CALLS, ids=lambda x: getattr(x, "__name__", ""))
def test_null_pointers_types_and_scales(fn, spec):
    names = dict(spec)
    optional = {"weights", "lse"} if fn is not L.jf_kv8_attn_weights else set()
    if fn in (L.jf_kv8_prefill_attn, L.jf_kv8_evict):  # (none needed at these sizes)
        optional.add("ws")
    for name in ("k", "v", "cu", "start", "bt", "q", "lens", "ws", "out", "lse", "w", "dst", "kept",
                 "kept_w"):
        if name in names and name not in optional:
            assert _call(fn, spec, {name: None}) == INVALID, name
    for name in ("k", "v", "q", "out", "ws"):
        if name in names:
            assert _call(fn, spec, {name: 24}) == INVALID, name
    if "dtype" in names:
        assert _call(fn, spec, {"dtype": 2}) == UNSUPPORTED
    if "scale" in names:
        for s in (NAN, INF, -INF):
            assert _call(fn, spec, {"scale": s}) == INVALID
    for name in ("B", "max_pages"):
        if name in names:
            assert _call(fn, spec, {name: 0}) == INVALID
            assert _call(fn, spec, {name: -3}) == INVALID
    assert _call(fn, spec, {"max_pages": 1 << 23}) == INVALID  # positions above 2^31


def test_append_sizes():
    assert _call(L.jf_kv8_append, APPEND, {"total": -1}) == INVALID
    assert _call(L.jf_kv8_append, APPEND, {"total": 0, "k": None}) == OK
    assert _call(L.jf_kv8_append, APPEND, {"total": (1 << 31) - 1, "layout": (256, 8, 128, 16, 4)}) == \
        UNSUPPORTED


def test_decode_sizes():
    for change, want in (({"hq": 30}, INVALID), ({"hq": 0}, INVALID), ({"sq": 0}, UNSUPPORTED),
                         ({"sq": 5}, UNSUPPORTED), ({"splits": 0}, INVALID),
                         ({"splits": 1025}, INVALID), ({"ws_bytes": 1000}, INVALID),
                         ({"B": 3000}, UNSUPPORTED),
                         ({"weights": 16, "stride": 1023}, INVALID), ({"weights": 18, "stride": 1024}, INVALID)):
        assert _call(L.jf_kv8_decode_attn, DECODE, change) == want, change
    lay = jfkv.layout(*LAY)
    plain = jfkv.jf_kv8_decode_workspace_bytes(lay, 2, 3, 32, 64)
    assert plain == jfkv.jf_decode_workspace_bytes(2, 96, 128, 64)
    sums = jfkv.jf_kv8_decode_workspace_bytes(lay, 2, 3, 32, 64, 4)
    assert sums == plain + 2 * 96 * 4 + 2 * 96 * 1024 * 4
    assert _call(L.jf_kv8_decode_attn, DECODE, {"B": 2, "sq": 3, "splits": 64, "weights": 16,
                                                "stride": 1024, "ws_bytes": sums - 1}) == INVALID
    with pytest.raises(jfkv.JfError):
        jfkv.jf_kv8_decode_workspace_bytes(lay, 1, 1, 32, 64, -1)
    assert L.jf_kv8_decode_workspace_bytes(ctypes.byref(lay), 1, 1, 32, 64, 0, None) == INVALID


@pytest.mark.parametrize("fn,spec", [CALLS[2], CALLS[3]], ids=["prefill", "weights"])
def test_chunk_sizes(fn, spec):
    for change, want in (({"T": -1}, INVALID), ({"prefix": -1}, INVALID), ({"hq": 30}, INVALID),
                         ({"prefix": 1009}, INVALID), ({"T": 1015}, INVALID),
                         ({"T": (1 << 31) - 5000, "prefix": 0}, UNSUPPORTED),
                         ({"prefix": (1 << 31) - 1}, INVALID)):
        assert _call(fn, spec, change) == want, change
    assert _call(fn, spec, {"T": 0, "q": None}) == OK
    assert _call(L.jf_kv8_attn_weights, WEIGHTS, {"stride": 25}) == INVALID


def test_prefill_workspace():
    lay = jfkv.layout(*LAY)
    need = jfkv.jf_kv8_prefill_workspace_bytes(lay, 16, 32, 100000)
    assert need > 0 and need % (16 * 32 * 132 * 4) == 0
    assert jfkv.jf_kv8_prefill_workspace_bytes(lay, 0, 32, 100000) == 0
    assert jfkv.jf_kv8_prefill_workspace_bytes(lay, 16, 32, 0) == 0
    assert _call(L.jf_kv8_prefill_attn, PREFILL, {"max_pages": 400, "prefix": 100000,
                                                  "ws_bytes": need - 1}) == INVALID
    assert b"workspace" in L.jf_last_error()


def test_evict_sizes():
    for change, want in (({"keep": 0}, INVALID), ({"recent": -1}, INVALID), ({"recent": 101}, INVALID),
                         ({"keep": 257}, INVALID), ({"dst_pages": 0}, INVALID),
                         ({"stride": 1023}, INVALID), ({"B": 70000}, UNSUPPORTED)):
        assert _call(L.jf_kv8_evict, EVICT, change) == want, change


def test_pool_bytes():
    assert jfkv.kv8_pool_bytes(jfkv.layout(256, 8, 128, 64, 10)) == (10 * 8 * 256 * 128, 10 * 8 * 4)
    with pytest.raises(jfkv.JfError):
        jfkv.kv8_pool_bytes(jfkv.layout(256, 8, 96, 64, 10))


def test_evict_counts_that_32_bits_do_not_hold():
    for change in ({"keep": 1 << 30, "dst_pages": 1 << 23},
                   {"layout": (256, 8, 128, 16, 16), "keep": 1 << 28, "dst_pages": 1 << 20,
                    "max_pages": 1 << 20, "stride": 1 << 28}):
        assert _call(L.jf_kv8_evict, EVICT, change) == UNSUPPORTED, change


@pytest.mark.parametrize("fn,spec", CALLS[1:4], ids=lambda x: getattr(x, "__name__", ""))
def test_scales_that_overflow_in_base_two(fn, spec):
    for scale in (3e38, -3e38, 2.0 ** 126):
        assert _call(fn, spec, {"scale": scale}) == INVALID
