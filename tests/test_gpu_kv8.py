"""The 8-bit cache on the GPU against its plain implementation in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import kv8 as ref
from paper_2609_17475_amd import jfkv
from tests.kv8_cases import (Pair, STALE, check_lse, check_out, check_weights, dtype_of, i32, rows,
                             tables_for, wide)

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------ append
@pytest.mark.parametrize("P,hkv,d,block,bf16,lens,prefix", [
    (64, 1, 64, 16, False, [1], 0),
    (64, 2, 64, 32, True, [130, 1, 0, 64], 0),
    (128, 3, 128, 16, False, [5, 200, 33], 0),
    (256, 2, 128, 64, False, [300, 77], 0),
    (256, 1, 256, 128, True, [257, 600], 0),
    (64, 2, 256, 64, False, [64, 63, 65], 0),
    (128, 2, 128, 128, False, [100, 28, 129], 51),
    (64, 1, 128, 16, True, [1, 1, 17, 40, 3], 23),
])
def test_append_is_bit_exact(P, hkv, d, block, bf16, lens, prefix):
    rng = np.random.default_rng(P + d + block + len(lens))
    total = [n + prefix for n in lens]
    pages = sum(-(-max(n, 1) // P) for n in total) + 2
    p = Pair(P, hkv, d, block, pages, bf16)
    tables, _ = tables_for(rng, P, total, pages)
    if prefix:
        p.fill(rng, [prefix] * len(lens), tables)
        assert not p.differing()
    n = sum(lens)
    k, v = rows(rng, n, hkv, d, bf16, 3.0), rows(rng, n, hkv, d, bf16, 0.01)
    p.append(k, v, np.cumsum([0] + lens).tolist(), [prefix] * len(lens), tables)
    assert not p.differing()


@pytest.mark.parametrize("d,block,bf16", [(64, 16, False), (128, 32, True), (256, 64, False), (128, 128, False)])
def test_append_row_by_row_grows_the_exponent(d, block, bf16):
    rng = np.random.default_rng(d)
    p = Pair(128, 2, d, block, 2, bf16)
    tables = np.array([[1, 0]], np.int32)
    for i in range(block + 9):
        size = float(np.exp(rng.uniform(-6, 6)))
        k, v = (rows(rng, 1, 2, d, bf16, size) for _ in range(2))
        p.append(k, v, [0, 1], [i], tables)
    assert not p.differing()


@pytest.mark.parametrize("bf16", [False, True])
def test_append_of_extreme_values(bf16):
    rng = np.random.default_rng(5)
    p = Pair(64, 1, 64, 16, 2, bf16)
    f = torch.finfo(dtype_of(bf16))
    k, v = (rows(rng, 64, 1, 64, bf16) for _ in range(2))
    k[:16] = 0.0
    k[16:32] *= f.tiny
    k[20, 0, 7] = -0.0
    k[32, 0, :3] = torch.tensor([f.max, -f.max, f.smallest_normal])
    k[48, 0, :4] = torch.tensor([float("inf"), -float("inf"), float("nan"), 448.0])
    v[:16] = float("nan")
    v[16:32, :, :] = float("inf")
    v[33] = f.smallest_normal / 4
    # values half way between two codes, at an exponent of 0
    v[48:64] = 1.0
    v[48, 0, :8] = torch.tensor([448.0, 17.0, 19.0, 21.0, -23.0, 2.0 ** -10, 3 * 2.0 ** -10, 1.0625])
    p.append(k, v, [0, 64], [0], np.array([[1]], np.int32))
    assert not p.differing()
    assert not np.any((p.host.codes[0] == 0x7F)[1]) and not np.any((p.host.codes[1] & 127 == 127)[1])


def test_append_skips_what_has_no_place():
    rng = np.random.default_rng(6)
    p = Pair(64, 1, 64, 16, 4)
    tables = np.array([[2, 9, 1], [-1, 0, -1], [3, -5, 1 << 30]], np.int32)
    lens, start = [150, 70, 90], [-20, 30, 120]
    k, v = (rows(rng, 310, 1, 64, False) for _ in range(2))
    p.append(k, v, [0, 150, 220, 310], start, tables)
    assert not p.differing()


def test_append_rewrites_after_a_rejected_draft():
    rng = np.random.default_rng(7)
    p = Pair(64, 2, 128, 32, 2)
    tables = np.array([[1, 0]], np.int32)
    p.fill(rng, [50], tables, 10.0)
    for start, n in ((47, 3), (47, 20), (32, 4), (0, 1)):
        k, v = (rows(rng, n, 2, 128, False) for _ in range(2))
        p.append(k, v, [0, n], [start], tables)
        assert not p.differing()


# ------------------------------------------------------------------ decode
def decode(p, q, tables, lens, scale, splits=64, ws=None, weights=None):
    B, sq, hq, d = q.shape
    if ws is None:
        ws = torch.zeros(jfkv.jf_kv8_decode_workspace_bytes(
            p.lay, B, sq, hq, splits, 0 if weights is None else tables.shape[1]), dtype=torch.uint8,
            device="cuda")
    out = torch.full(q.shape, float("nan"), dtype=q.dtype, device="cuda")
    jfkv.jf_kv8_decode_attn(p.gpu, q.cuda(), i32(tables), i32(lens), scale, splits, ws, out,
                            weights=weights)
    torch.cuda.synchronize()
    assert not ws[:262144].any()
    return out


DECODE = [
    # P, hkv, hq, d, block, bf16, lens, sq, splits
    (64, 1, 1, 64, 16, False, [1], 1, 64),
    (64, 1, 4, 128, 64, False, [33, 0, 64, 65], 1, 64),
    (64, 2, 8, 128, 16, True, [700, 31, 257], 1, 8),
    (256, 2, 14, 64, 32, False, [1000, 513], 1, 3),
    (128, 1, 6, 256, 32, True, [900, 40], 3, 64),
    (128, 2, 8, 128, 128, False, [1500], 4, 64),
    (64, 1, 24, 64, 16, False, [300, 3, 2], 4, 64),   # 96 pairs: six column chunks
    (256, 3, 15, 128, 64, True, [2100, 1], 2, 1),
    (64, 1, 40, 256, 64, False, [130], 1, 64),
    (64, 8, 8, 128, 64, False, [5000], 1, 1024),
]


@pytest.mark.parametrize("P,hkv,hq,d,block,bf16,lens,sq,splits", DECODE)
@pytest.mark.parametrize("sums", [False, True])
def test_decode(P, hkv, hq, d, block, bf16, lens, sq, splits, sums):
    rng = np.random.default_rng(hq + d + len(lens))
    pages = sum(-(-max(n, 1) // P) for n in lens) + 1
    p = Pair(P, hkv, d, block, pages, bf16)
    tables, _ = tables_for(rng, P, lens, pages)
    p.fill(rng, lens, tables)
    q = rows(rng, len(lens) * sq, hq, d, bf16, 0.7).view(len(lens), sq, hq, d)
    scale = d ** -0.5
    cap = tables.shape[1] * P
    w = before = None
    if sums:
        before = rng.random((len(lens), hkv, cap + 3)).astype(np.float32)
        w = torch.from_numpy(before).cuda()
    out = decode(p, q, tables, lens, scale, splits, weights=w)
    for b, n in enumerate(lens):
        r = ref.attend(p.host, wide(q[b]), tables[b], n, scale)
        check_out(out[b], r, d, bf16, "request %d" % b)
        if sums:
            got = w[b].cpu().numpy()
            check_weights(got[:, :n], before[b, :, :n], r["weights"], r, d, n, sq * hq // hkv)
            assert np.array_equal(got[:, n:], before[b, :, n:])  # behind the request


def test_decode_of_one_request_is_the_same_in_any_batch():
    rng = np.random.default_rng(1)
    lens = [777, 64, 1301]
    p = Pair(64, 2, 128, 32, 40)
    tables, _ = tables_for(rng, 64, lens, 40)
    p.fill(rng, lens, tables)
    q = rows(rng, 3, 8, 128, False).view(3, 1, 8, 128)
    whole = decode(p, q, tables, lens, 0.1)
    again = decode(p, q, tables, lens, 0.1)
    assert torch.equal(whole, again)
    for b in range(3):
        assert torch.equal(decode(p, q[b:b + 1], tables[b:b + 1], lens[b:b + 1], 0.1)[0], whole[b])


@pytest.mark.parametrize("hq,d,block,bf16,sq", [(4, 128, 64, False, 1), (2, 64, 16, True, 1),
                                                (4, 256, 32, True, 1), (6, 256, 64, False, 3),
                                                (9, 128, 32, False, 2), (5, 64, 64, False, 4)])
def test_decode_of_many_splits_alone_and_in_a_batch(hq, d, block, bf16, sq):
    """Requests of more than 16 splits, of one and of none; the same bits alone."""
    rng = np.random.default_rng(hq * sq)
    lens = [3601, 0, 90, 2900]
    p = Pair(128, 1, d, block, 60, bf16)
    tables, _ = tables_for(rng, 128, lens, 60)
    p.fill(rng, lens, tables)
    q = rows(rng, 4 * sq, hq, d, bf16, 0.7).view(4, sq, hq, d)
    cap = tables.shape[1] * 128
    w = torch.zeros(4, 1, cap, device="cuda")
    out = decode(p, q, tables, lens, d ** -0.5, weights=w)
    for b, n in enumerate(lens):
        r = ref.attend(p.host, wide(q[b]), tables[b], n, d ** -0.5)
        check_out(out[b], r, d, bf16, "request %d" % b)
        check_weights(w[b, :, :n].cpu().numpy(), np.zeros((1, n), np.float32), r["weights"], r, d, n,
                      sq * hq)
        w1 = torch.zeros(1, 1, cap, device="cuda")
        alone = decode(p, q[b:b + 1], tables[b:b + 1], lens[b:b + 1], d ** -0.5, weights=w1)
        assert torch.equal(alone[0], out[b]) and torch.equal(w1[0], w[b])


@pytest.mark.parametrize("scale", [0.3, -0.3, 0.0, 1e-30])
def test_decode_scales(scale):
    rng = np.random.default_rng(2)
    p = Pair(64, 1, 64, 16, 4)
    tables, _ = tables_for(rng, 64, [200], 4)
    p.fill(rng, [200], tables)
    q = rows(rng, 1, 2, 64, False).view(1, 1, 2, 64)
    check_out(decode(p, q, tables, [200], scale)[0], ref.attend(p.host, wide(q[0]), tables[0], 200, scale), 64, False)


def test_decode_lengths_outside_the_table():
    rng = np.random.default_rng(3)
    p = Pair(64, 1, 64, 16, 4)
    tables = np.array([[0, 1], [2, 3]], np.int32)
    p.fill(rng, [128, 128], tables)
    q = rows(rng, 2, 2, 64, False).view(2, 1, 2, 64)
    w = torch.zeros(2, 1, 128, device="cuda")
    out = decode(p, q, tables, [5000, -7], 0.2, weights=w)
    check_out(out[0], ref.attend(p.host, wide(q[0]), tables[0], 128, 0.2), 64, False)
    assert not out[1].any() and not w[1].any()


def test_decode_passes_over_pages_outside_the_pool():
    rng = np.random.default_rng(4)
    p = Pair(64, 2, 128, 32, 6)
    tables = np.array([[3, 1, 5, 0]], np.int32)
    p.fill(rng, [230], tables)
    bad = tables.copy()
    bad[0, 1], bad[0, 3] = 6, -1
    q = rows(rng, 2, 4, 128, False).view(1, 2, 4, 128)
    before = rng.random((1, 2, 256)).astype(np.float32)
    w = torch.from_numpy(before).cuda()
    out = decode(p, q, bad, [230], 0.1, weights=w)
    r = ref.attend(p.host, wide(q[0]), bad[0], 230, 0.1)
    check_out(out[0], r, 128, False)
    check_weights(w[0].cpu().numpy()[:, :230], before[0, :, :230], r["weights"], r, 128, 230, 4)
    none = np.full_like(tables, -1)
    assert not decode(p, q, none, [230], 0.1).any()


@pytest.mark.parametrize("d,bf16", [(64, False), (128, True), (256, False)])
@pytest.mark.parametrize("block", [16, 64])
def test_decode_where_exponents_jump(d, bf16, block):
    """Blocks whose values differ by up to 2^24: no common reference holds them."""
    rng = np.random.default_rng(d + block)
    n = 420
    p = Pair(64, 1, d, block, 7, bf16)
    tables, _ = tables_for(rng, 64, [n], 7)
    size = np.exp2(rng.integers(-12, 13, -(-n // 16))).repeat(16)[:n, None, None]
    k = rows(rng, n, 1, d, bf16)
    v = (rows(rng, n, 1, d, False).double() * torch.from_numpy(size)).to(dtype_of(bf16))
    p.append(k, v, [0, n], [0], tables)
    q = rows(rng, 3, 4, d, bf16, 2.0).view(1, 3, 4, d)
    check_out(decode(p, q, tables, [n], d ** -0.5)[0], ref.attend(p.host, wide(q[0]), tables[0], n, d ** -0.5),
              d, bf16)
    # and a needle: all weight on a position whose values are the smallest
    v[:] = v.abs() + 1
    v[100:104] = 2.0 ** -12
    k[100] = 8.0
    p.append(k, v, [0, n], [0], tables)
    q = torch.ones(1, 1, 2, d, dtype=dtype_of(bf16))
    check_out(decode(p, q, tables, [n], 1.0)[0], ref.attend(p.host, wide(q[0]), tables[0], n, 1.0), d, bf16)


def test_decode_of_growing_and_shrinking_scores():
    rng = np.random.default_rng(8)
    n = 600
    for sign in (1.0, -1.0):
        p = Pair(64, 1, 64, 16, 10)
        tables, _ = tables_for(rng, 64, [n], 10)
        k, v = (rows(rng, n, 1, 64, False) for _ in range(2))
        k[:, 0, 0] = torch.linspace(-200, 200, n) * sign
        p.append(k, v, [0, n], [0], tables)
        q = rows(rng, 1, 3, 64, False).view(1, 1, 3, 64)
        q[..., 0] = 1.0
        check_out(decode(p, q, tables, [n], 1.0)[0], ref.attend(p.host, wide(q[0]), tables[0], n, 1.0), 64, False)


# ------------------------------------------------------------------ chunks
def prefill(p, q, table, prefix, scale, split=True):
    T, hq, d = q.shape
    out = torch.full(q.shape, float("nan"), dtype=q.dtype, device="cuda")
    lse = torch.full((T, hq), float("nan"), device="cuda")
    ws = None
    if split:
        ws = torch.full((jfkv.jf_kv8_prefill_workspace_bytes(p.lay, T, hq, prefix),), 0xFF,
                        dtype=torch.uint8, device="cuda")
    jfkv.jf_kv8_prefill_attn(p.gpu, q.cuda(), i32(table), prefix, scale, out, lse=lse, workspace=ws)
    torch.cuda.synchronize()
    return out, lse


CHUNKS = [
    # P, hkv, hq, d, block, bf16, T, prefix
    (64, 1, 1, 64, 16, False, 1, 0),
    (64, 1, 4, 128, 64, False, 1, 64),
    (64, 2, 6, 128, 16, True, 65, 0),
    (256, 1, 4, 128, 64, False, 70, 500),
    (128, 2, 4, 256, 32, True, 50, 333),
    (64, 1, 7, 64, 32, False, 130, 61),
    (128, 1, 16, 256, 128, False, 17, 1000),
    (64, 3, 3, 64, 64, True, 300, 3),
    (256, 1, 2, 128, 32, False, 3, 2500),
    (64, 2, 24, 128, 16, False, 40, 200),
    (256, 8, 8, 64, 64, True, 5, 13000),   # few columns over many positions
    (256, 8, 8, 128, 128, False, 6, 12500),
]


@pytest.mark.parametrize("P,hkv,hq,d,block,bf16,T,prefix", CHUNKS)
def test_prefill_and_its_weights(P, hkv, hq, d, block, bf16, T, prefix):
    rng = np.random.default_rng(T + prefix)
    n = T + prefix
    pages = -(-n // P) + 1
    p = Pair(P, hkv, d, block, pages, bf16)
    tables, _ = tables_for(rng, P, [n], pages)
    p.fill(rng, [n], tables)
    q = rows(rng, T, hq, d, bf16, 0.7)
    scale = d ** -0.5
    r = ref.attend(p.host, wide(q), tables[0], n, scale)
    for split in (False, True):
        out, lse = prefill(p, q, tables[0], prefix, scale, split)
        check_out(out, r, d, bf16, "split %s" % split)
        check_lse(lse, r, d, n)
    before = rng.random((hkv, n + 5)).astype(np.float32)
    w = torch.from_numpy(before).cuda()
    jfkv.jf_kv8_attn_weights(p.gpu, q.cuda(), lse, i32(tables[0]), prefix, scale, w)
    got = w.cpu().numpy()
    r["dots"] *= 2  # (the lse's own error beside the scores')
    check_weights(got[:, :n], before[:, :n], r["weights"], r, d, n, T * hq // hkv)
    assert np.array_equal(got[:, n:], before[:, n:])
    again = torch.from_numpy(before).cuda()
    jfkv.jf_kv8_attn_weights(p.gpu, q.cuda(), lse, i32(tables[0]), prefix, scale, again)
    assert torch.equal(w, again)
    # the last rows alone, as a window
    if T > 4:
        part = torch.zeros(hkv, n, device="cuda")
        jfkv.jf_kv8_attn_weights(p.gpu, q[T - 3:].contiguous().cuda(), lse[T - 3:], i32(tables[0]),
                                 n - 3, scale, part)
        rw = ref.attend(p.host, wide(q[T - 3:]), tables[0], n, scale)
        rw["dots"] *= 2
        check_weights(part.cpu().numpy(), np.zeros((hkv, n)), rw["weights"], rw, d, n, 3 * hq // hkv)


def window(host, q, table, n, scale, first):
    """As ref.attend, all rows of a head at once: lse, the weights that rows first ..
    add, and the largest scale * sum |q k|."""
    T, hq, d = q.shape
    g = hq // host.hkv
    lse, weights, dots = np.empty((T, hq)), np.zeros((host.hkv, n)), 0.0
    sees = np.arange(n)[:, None] <= n - T + np.arange(T)[None, :]
    for h in range(host.hkv):
        k, ok = host.values(0, table, n, h)
        k = np.where(ok[:, None], k, 0.0)
        for j in range(h * g, h * g + g):
            z = np.where(sees & ok[:, None], scale * (k @ q[:, j].T), -np.inf)
            dots = max(dots, float(np.max(abs(scale) * (np.abs(k) @ np.abs(q[:, j]).T))))
            top = z.max(0)
            lse[:, j] = top + np.log(np.exp(z - top).sum(0))
            weights[h] += np.exp(z - lse[:, j])[:, first:].sum(1)
    return lse, weights, dots


@pytest.mark.parametrize("P,hkv,hq,d,block,bf16,T,n,scale", [
    (256, 8, 16, 128, 64, False, 3, 16301, 0.05),     # one pair of column groups
    (256, 8, 16, 128, 32, True, 37, 16384, 0.05),     # three, the last half empty
    (64, 3, 9, 128, 16, False, 64, 42331, -0.05),     # heads that the chip's count is no multiple of
    (256, 16, 48, 256, 32, True, 11, 16140, 0.03),
])
def test_weights_of_a_window_over_many_positions(P, hkv, hq, d, block, bf16, T, n, scale):
    rng = np.random.default_rng(n)
    pages = -(-n // P) + 2
    p = Pair(P, hkv, d, block, pages, bf16)
    for which in range(2):
        c = rng.integers(0, 256, p.host.codes[which].shape, np.uint8)
        c[(c & 127) == 127] = 0
        p.host.codes[which][...] = c
        p.host.exps[which][...] = rng.integers(117, 121, p.host.exps[which].shape)
    tables, _ = tables_for(rng, P, [n], pages)
    tables[0, 5] = pages
    page, slot = tables[0, (n - 1) // P], (n - 1) % P + 1
    p.host.codes[0][page, :, slot:] = STALE  # slots not written yet
    for name, data in zip(("k_codes", "k_exps", "v_codes", "v_exps"), p.host.pool_bytes()):
        getattr(p.gpu, name).copy_(torch.from_numpy(np.ascontiguousarray(data)))
    q = rows(rng, T, hq, d, bf16, 0.3)
    before = rng.random((hkv, n + 3)).astype(np.float32)
    for hidden in (0, 1):  # (rows that saw nothing add nothing)
        z, added, dots = window(p.host, wide(q), tables[0], n, scale, hidden)
        lse = torch.from_numpy(z.astype(np.float32)).cuda()
        lse[:hidden] = -float("inf")
        w = torch.from_numpy(before).cuda()
        jfkv.jf_kv8_attn_weights(p.gpu, q.cuda(), lse, i32(tables[0]), n - T, scale, w)
        got = w.cpu().numpy()
        # (twice the scores' error: the lse's own rounding beside it)
        check_weights(got[:, :n], before[:, :n], added, dict(dots=2 * dots), d, n, T * hq // hkv)
        assert np.array_equal(got[:, n:], before[:, n:])
        assert np.array_equal(got[:, 5 * P:6 * P], before[:, 5 * P:6 * P])
        again = torch.from_numpy(before).cuda()
        jfkv.jf_kv8_attn_weights(p.gpu, q.cuda(), lse, i32(tables[0]), n - T, scale, again)
        assert torch.equal(w, again)


@pytest.mark.parametrize("split", [False, True])
def test_prefill_passes_over_pages_outside_the_pool(split):
    rng = np.random.default_rng(4)
    p = Pair(64, 2, 128, 32, 8)
    tables = np.array([[3, 1, 5, 0, 7, 2]], np.int32)
    p.fill(rng, [380], tables)
    bad = tables[0].copy()
    bad[0], bad[3] = 8, -1
    q = rows(rng, 380, 4, 128, False)
    out, lse = prefill(p, q, bad, 0, 0.1, split)
    r = ref.attend(p.host, wide(q), bad, 380, 0.1)
    assert np.isneginf(r["lse"][:64]).all() and not out[:64].any()  # rows that see nothing
    check_out(out, r, 128, False)
    check_lse(lse, r, 128, 380)
    before = rng.random((2, 380)).astype(np.float32)
    w = torch.from_numpy(before).cuda()
    jfkv.jf_kv8_attn_weights(p.gpu, q.cuda(), lse, i32(bad), 0, 0.1, w)
    r["dots"] *= 2
    check_weights(w.cpu().numpy(), before, r["weights"], r, 128, 380, 760)
    assert np.array_equal(w.cpu().numpy()[:, :64], before[:, :64])


@pytest.mark.parametrize("scale", [-0.3, 0.0])
def test_prefill_scales(scale):
    rng = np.random.default_rng(9)
    p = Pair(64, 1, 64, 16, 4)
    tables, _ = tables_for(rng, 64, [200], 4)
    p.fill(rng, [200], tables)
    q = rows(rng, 100, 2, 64, False)
    r = ref.attend(p.host, wide(q), tables[0], 200, scale)
    out, lse = prefill(p, q, tables[0], 100, scale)
    check_out(out, r, 64, False)
    check_lse(lse, r, 64, 200)


@pytest.mark.parametrize("d,bf16,block", [(64, False, 16), (128, True, 16), (256, False, 64)])
def test_prefill_where_exponents_jump(d, bf16, block):
    rng = np.random.default_rng(d + block)
    n = 300
    p = Pair(64, 1, d, block, 5, bf16)
    tables, _ = tables_for(rng, 64, [n], 5)
    size = np.exp2(rng.integers(-12, 13, -(-n // 16))).repeat(16)[:n, None, None]
    k = rows(rng, n, 1, d, bf16)
    v = (rows(rng, n, 1, d, False).double() * torch.from_numpy(size)).to(dtype_of(bf16))
    p.append(k, v, [0, n], [0], tables)
    q = rows(rng, 200, 2, d, bf16, 2.0)
    out, lse = prefill(p, q, tables[0], 100, d ** -0.5)
    check_out(out, ref.attend(p.host, wide(q), tables[0], n, d ** -0.5), d, bf16)


# ------------------------------------------------------------------ eviction
def evict(p, tables, lens, w, keep, recent, dst):
    B, hkv = len(lens), p.lay.num_kv_heads
    kept = torch.full((B, hkv, keep), 77, dtype=torch.int32, device="cuda")
    kept_w = torch.full((B, hkv, keep), 77.0, device="cuda")
    ws = torch.full((jfkv.jf_kv8_evict_workspace_bytes(p.lay, B, tables.shape[1], keep),), 0xFF,
                    dtype=torch.uint8, device="cuda")
    jfkv.jf_kv8_evict(p.gpu, i32(tables), i32(lens), torch.from_numpy(w).cuda(), keep, recent,
                      i32(dst), ws, kept, kept_w)
    want, want_w = ref.evict(p.host, tables, lens, w, keep, recent, dst)
    assert np.array_equal(kept.cpu().numpy(), want)
    assert np.array_equal(kept_w.cpu().numpy(), want_w, equal_nan=True)
    assert not p.differing()
    return want


@pytest.mark.parametrize("P,hkv,d,block,lens,keep,recent", [
    (64, 1, 64, 16, [1], 1, 0),
    (64, 2, 128, 32, [200, 37, 0, 64], 50, 10),
    (128, 1, 256, 128, [700], 300, 0),
    (64, 3, 64, 64, [130, 129], 128, 128),
    (256, 2, 128, 64, [3000, 2999], 600, 33),
    (64, 1, 64, 16, [90], 200, 40),
    (64, 2, 128, 16, [5000], 17, 1),
    (256, 2, 64, 128, [20000, 300, 16385], 5000, 100),
    (256, 1, 64, 64, [33000], 17, 0),
])
@pytest.mark.parametrize("kind", ["spread", "equal", "odd"])
def test_evict(P, hkv, d, block, lens, keep, recent, kind):
    rng = np.random.default_rng(keep + len(lens))
    more = -(-keep // P)
    pages = sum(-(-max(n, 1) // P) for n in lens) + more * len(lens) + 1
    p = Pair(P, hkv, d, block, pages)
    tables, rest = tables_for(rng, P, lens, pages)
    dst = rest[:more * len(lens)].reshape(len(lens), more).astype(np.int32)
    n = sum(lens)
    size = np.exp2(rng.integers(-8, 5, n))[:, None, None]
    k, v = ((rows(rng, n, hkv, d, False).double() * torch.from_numpy(size)).half() for _ in range(2))
    p.append(k, v, np.cumsum([0] + lens).tolist(), [0] * len(lens), tables)
    w = rng.random((len(lens), hkv, tables.shape[1] * P + 2)).astype(np.float32) ** 8
    if kind == "equal":
        w = np.round(w * 3).astype(np.float32)
    elif kind == "odd":
        w[rng.random(w.shape) < 0.1] = np.nan
        w[rng.random(w.shape) < 0.1] = np.inf
        w[rng.random(w.shape) < 0.2] = -0.0
        w[rng.random(w.shape) < 0.2] *= -1
        w[rng.random(w.shape) < 0.05] = -np.inf
        w[rng.random(w.shape) < 0.05] = 1e-42
    evict(p, tables, lens, w, keep, recent, dst)


def test_evict_passes_over_pages_outside_the_pool():
    rng = np.random.default_rng(3)
    p = Pair(64, 1, 64, 16, 8)
    tables = np.array([[0, 1, 2]], np.int32)
    p.fill(rng, [190], tables)
    w = rng.random((1, 1, 192)).astype(np.float32)
    evict(p, np.array([[0, 9, 2]], np.int32), [190], w, 100, 5, np.array([[5, -1]], np.int32))


# ------------------------------------------------------------------ together
def test_a_session_with_eviction():
    """Prompt, its weights, steps that add theirs, eviction, steps over the shorter cache."""
    rng = np.random.default_rng(11)
    P, hkv, hq, d, keep = 64, 2, 8, 128, 96
    p = Pair(P, hkv, d, 32, 16)
    perm = rng.permutation(16).astype(np.int32)
    table, dst = perm[None, :6], perm[None, 6:8]
    n = 300
    scale = d ** -0.5
    p.fill(rng, [n], table)
    q = rows(rng, 120, hq, d, False)
    out, lse = prefill(p, q, table[0], n - 120, scale)
    r = ref.attend(p.host, wide(q), table[0], n, scale)
    check_out(out, r, d, False)
    w = torch.zeros(1, hkv, 6 * P, device="cuda")
    jfkv.jf_kv8_attn_weights(p.gpu, q.cuda(), lse, i32(table[0]), n - 120, scale, w[0])
    total = r["weights"].copy()
    for step in range(5):
        k, v = (rows(rng, 1, hkv, d, False) for _ in range(2))
        p.append(k, v, [0, 1], [n], table)
        n += 1
        q1 = rows(rng, 1, hq, d, False).view(1, 1, hq, d)
        out = decode(p, q1, table, [n], scale, weights=w)
        r = ref.attend(p.host, wide(q1[0]), table[0], n, scale)
        check_out(out[0], r, d, False)
        total = np.pad(total, ((0, 0), (0, 1))) + r["weights"]
    got = w.cpu().numpy()
    assert np.allclose(got[0, :, :n], total, rtol=1e-4, atol=1e-6)
    kept = evict(p, table, [n], got, keep, 20, dst)
    assert (kept[0, :, -20:] == np.arange(n - 20, n)).all()
    n = keep
    for step in range(6):
        k, v = (rows(rng, 1, hkv, d, False) for _ in range(2))
        p.append(k, v, [0, 1], [n], dst)
        n += 1
        q1 = rows(rng, 1, hq, d, False).view(1, 1, hq, d)
        check_out(decode(p, q1, dst, [n], scale)[0], ref.attend(p.host, wide(q1[0]), dst[0], n, scale), d, False)
        assert not p.differing()


def test_captured_step_replays_like_the_eager_one():
    """Append, decode with sums, prefill, weights and eviction in one graph; two
    graphs of different shapes share the workspaces, one after the other."""
    rng = np.random.default_rng(12)
    P, hkv, hq, d, n, keep = 64, 2, 8, 128, 500, 100
    side = torch.cuda.Stream()
    ws = torch.zeros(1 << 24, dtype=torch.uint8, device="cuda")
    more = torch.zeros(1 << 24, dtype=torch.uint8, device="cuda")

    def build(bf16, seed):
        rng = np.random.default_rng(seed)
        p = Pair(P, hkv, d, 32, 12, bf16)
        table = np.arange(8, dtype=np.int32)[None]
        p.fill(rng, [n], table)
        k, v = (rows(rng, 1, hkv, d, bf16).cuda() for _ in range(2))
        q = rows(rng, 1, hq, d, bf16).view(1, 1, hq, d).cuda()
        qs = rows(rng, 40, hq, d, bf16).cuda()
        out, outs = torch.empty_like(q), torch.empty_like(qs)
        lse = torch.empty(40, hq, device="cuda")
        w = torch.zeros(1, hkv, 8 * P, device="cuda")
        kept = torch.empty(1, hkv, keep, dtype=torch.int32, device="cuda")
        kept_w = torch.empty(1, hkv, keep, device="cuda")
        t, dst, lens = i32(table), i32([[9, 10]]), i32([n + 1])
        s = dict(stream=side)
        calls = [jfkv.bind_kv8_append(p.gpu, k, v, i32([0, 1]), i32([n]), t, **s),
                 jfkv.bind_kv8_decode(p.gpu, q, t, lens, 0.1, 64, ws, out, weights=w, **s),
                 jfkv.bind_kv8_prefill(p.gpu, qs, t[0], n - 39, 0.1, outs, lse=lse, workspace=more, **s),
                 jfkv.bind_kv8_attn_weights(p.gpu, qs, lse, t[0], n - 39, 0.1, w[0], **s),
                 jfkv.bind_kv8_evict(p.gpu, t, lens, w, keep, 10, dst, more, kept, kept_w, **s)]
        return p, calls, w, (out, outs, lse, w, kept, kept_w, p.gpu.k_codes, p.gpu.v_codes, p.gpu.k_exps)

    graphs = []
    for bf16 in (False, True):
        p, calls, w, results = build(bf16, 20 + bf16)
        with torch.cuda.stream(side):
            for c in calls:
                c()
            side.synchronize()
            want = [t.clone() for t in results]
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=side):
                w.zero_()
                for c in calls:
                    c()
        graphs.append((g, calls, w, results, want, p))
    for turn in range(3):
        for g, calls, w, results, want, p in graphs:
            for t in results[:6]:
                t.fill_(1)
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            for a, b in zip(results, want):
                assert torch.equal(a, b)
            with torch.cuda.stream(side):  # the program's own eager work between replays
                w.zero_()
                for c in calls:
                    c()
            torch.cuda.synchronize()
            for a, b in zip(results, want):
                assert torch.equal(a, b)


def random_pool(rng, P, hkv, d, block, pages):
    """A pool of random finite codes and small exponents, unlike any appended one."""
    pool = jfkv.KV8Pool(jfkv.layout(P, hkv, d, block, pages))
    for t in (pool.k_codes, pool.v_codes):
        c = rng.integers(0, 256, t.numel(), np.uint8)
        c[(c & 127) == 127] = 0
        t.copy_(torch.from_numpy(c))
    for t in (pool.k_exps, pool.v_exps):
        t.copy_(torch.from_numpy(rng.integers(117, 121, t.numel()).astype(np.uint8)))
    return pool


def long_calls(pool, rng, P, hkv, hq, d, n, keep, dst, stream=None):
    """Calls that take the larger launches (records joined apart, eviction in parts,
    a window's weights where the chip is filled), and what they write."""
    s = dict(stream=stream)
    pages = -(-n // P)
    t, lens = i32(np.stack([np.arange(pages), np.arange(pages)[::-1]])), i32([n, n - 77])
    q = rows(rng, 6, hq, d, True, 0.5).view(2, 3, hq, d).cuda()
    qs = rows(rng, 9, hq, d, True, 0.5).cuda()
    out, outs = torch.empty_like(q), torch.empty_like(qs)
    lse = torch.empty(9, hq, device="cuda")
    w = torch.zeros(2, hkv, pages * P, device="cuda")
    kept = torch.empty(2, hkv, keep, dtype=torch.int32, device="cuda")
    kept_w = torch.empty(2, hkv, keep, device="cuda")
    ws = torch.zeros(jfkv.jf_kv8_decode_workspace_bytes(pool.layout, 2, 3, hq, 64, pages),
                     dtype=torch.uint8, device="cuda")
    ws2, ws3 = (torch.empty(max(16, b), dtype=torch.uint8, device="cuda") for b in (
        jfkv.jf_kv8_prefill_workspace_bytes(pool.layout, 9, hq, n - 9),
        jfkv.jf_kv8_evict_workspace_bytes(pool.layout, 2, pages, keep)))
    calls = [jfkv.bind_kv8_decode(pool, q, t, lens, 0.03, 64, ws, out, weights=w, **s),
             jfkv.bind_kv8_prefill(pool, qs, t[0], n - 9, 0.03, outs, lse=lse, workspace=ws2, **s),
             jfkv.bind_kv8_attn_weights(pool, qs, lse, t[0], n - 9, 0.03, w[0], **s),
             jfkv.bind_kv8_evict(pool, t, lens, w, keep, 50, i32(dst), ws3, kept, kept_w, **s)]
    return calls, w, (out, outs, lse, w, kept, kept_w)


def dst_bytes(pool, pages):
    lay = pool.layout
    n = lay.num_kv_heads * lay.page_size
    return [t.view(-1, n * lay.head_dim // per)[pages].clone() for t, per in (
        (pool.k_codes, 1), (pool.v_codes, 1), (pool.k_exps, lay.head_dim * lay.group_size),
        (pool.v_exps, lay.head_dim * lay.group_size))]


@pytest.mark.parametrize("d,hkv,hq", [(256, 8, 48), (128, 8, 56)])
def test_captured_long_calls_replay_like_eager_ones(d, hkv, hq):
    rng = np.random.default_rng(d)
    P, n, keep = 256, 33000 if d > 128 else 17000, 700
    pages = -(-n // P)
    pool = random_pool(rng, P, hkv, d, 32, pages + 6)
    dst = np.arange(pages, pages + 6).reshape(2, 3)
    side = torch.cuda.Stream()
    calls, w, results = long_calls(pool, rng, P, hkv, hq, d, n, keep, dst, side)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for c in calls:
            c()
        side.synchronize()
        want = [t.clone() for t in results] + dst_bytes(pool, slice(pages, None))
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            w.zero_()
            for c in calls:
                c()
    for turn in range(3):
        for run in (g.replay, None):
            for t in results:
                t.fill_(1)
            torch.cuda.synchronize()
            if run:
                run()
            else:
                with torch.cuda.stream(side):
                    w.zero_()
                    for c in calls:
                        c()
            torch.cuda.synchronize()
            for a, b in zip(list(results) + dst_bytes(pool, slice(pages, None)), want):
                assert torch.equal(a, b)


def test_two_sets_of_calls_at_once():
    """Two streams over one pool, each with its own workspaces and pages to move to."""
    rng = np.random.default_rng(6)
    P, hkv, hq, d, n, keep = 256, 8, 48, 128, 17000, 700
    pages = -(-n // P)
    pool = random_pool(rng, P, hkv, d, 64, pages + 12)
    streams = [torch.cuda.Stream() for _ in range(2)]
    sets = [long_calls(pool, rng, P, hkv, hq, d, n, keep,
                       np.arange(pages + 6 * i, pages + 6 * i + 6).reshape(2, 3), st)
            for i, st in enumerate(streams)]
    torch.cuda.synchronize()
    want = None
    for alone in (True, False, False):
        for (calls, w, results), st in zip(sets, streams):
            w.zero_()
        torch.cuda.synchronize()
        for i in range(len(sets[0][0])):
            for calls, w, results in sets:
                calls[i]()
                if alone:
                    torch.cuda.synchronize()
        torch.cuda.synchronize()
        got = [t.clone() for _, _, r in sets for t in r] + dst_bytes(pool, slice(pages, None))
        if want is None:
            want = got
        for a, b in zip(got, want):
            assert torch.equal(a, b)


def test_pages_beyond_four_gibibytes():
    """The last pages of a pool whose arrays pass 2^32 bytes, against a small pool."""
    rng = np.random.default_rng(8)
    P, hkv, hq, d, block = 1024, 8, 16, 256, 64
    small = random_pool(rng, P, hkv, d, block, 8)
    first = (1 << 32) // (P * hkv * d) + 3
    big = jfkv.KV8Pool(jfkv.layout(P, hkv, d, block, first + 8))
    for name in ("k_codes", "k_exps", "v_codes", "v_exps"):
        a, b = getattr(small, name), getattr(big, name)
        b[b.numel() - a.numel():].copy_(a)
    n = 5 * P + 100
    k, v = (rows(rng, 200, hkv, d, True).cuda() for _ in range(2))
    q = rows(rng, 2, hq, d, True, 0.3).view(1, 2, hq, d).cuda()
    qs = rows(rng, 70, hq, d, True, 0.3).cuda()
    w0 = torch.from_numpy(rng.random((1, hkv, 6 * P)).astype(np.float32)).cuda()
    got = []
    for pool, at in ((small, 0), (big, first)):
        t, dst = i32([[at + i for i in (4, 0, 5, 2, 1, 3)]]), i32([[at + 7, at + 6]])
        jfkv.jf_kv8_append(pool, k, v, i32([0, 200]), i32([n - 200]), t)
        w = w0.clone()
        ws = torch.zeros(jfkv.jf_kv8_decode_workspace_bytes(pool.layout, 1, 2, hq, 64, 6),
                         dtype=torch.uint8, device="cuda")
        out, outs, lse = torch.empty_like(q), torch.empty_like(qs), torch.empty(70, hq, device="cuda")
        jfkv.jf_kv8_decode_attn(pool, q, t, i32([n]), 0.03, 64, ws, out, weights=w)
        jfkv.jf_kv8_prefill_attn(pool, qs, t[0], n - 70, 0.03, outs, lse=lse)
        jfkv.jf_kv8_attn_weights(pool, qs, lse, t[0], n - 70, 0.03, w[0])
        kept = torch.empty(1, hkv, 1500, dtype=torch.int32, device="cuda")
        kept_w = torch.empty(1, hkv, 1500, device="cuda")
        jfkv.jf_kv8_evict(pool, t, i32([n]), w, 1500, 64, dst, None, kept, kept_w)
        got.append([out, outs, lse, w, kept, kept_w] + dst_bytes(pool, slice(at, None)))
    torch.cuda.synchronize()
    assert torch.isfinite(got[0][0]).all() and got[0][0].any()
    for a, b in zip(*got):
        assert torch.equal(a, b)


def test_python_refusals():
    p = Pair(64, 2, 64, 16, 2)
    q = torch.zeros(1, 1, 4, 64, dtype=torch.float16, device="cuda")
    t, lens = i32([[0, 1]]), i32([5])
    ws = torch.zeros(1 << 22, dtype=torch.uint8, device="cuda")

    def call(q=q, t=t, lens=lens, out=None, w=None):
        jfkv.jf_kv8_decode_attn(p.gpu, q, t, lens, 1.0, 8, ws, torch.empty_like(q) if out is None else out,
                                weights=w)
    call()
    for kw in (dict(q=q.float()), dict(q=q.cpu()), dict(q=q[0]), dict(q=torch.zeros(1, 1, 4, 128, device="cuda").half()[..., ::2]),
               dict(out=q.bfloat16()), dict(out=q[..., :32]), dict(t=t.long()), dict(t=t[0]),
               dict(lens=lens.repeat(2)), dict(w=torch.zeros(1, 1, 128, device="cuda")),
               dict(w=torch.zeros(1, 2, 128, device="cuda").double())):
        with pytest.raises(ValueError):
            call(**kw)
    with pytest.raises(jfkv.JfError):
        call(w=torch.zeros(1, 2, 127, device="cuda"))
    with pytest.raises(ValueError):
        jfkv.KV8Pool(p.lay, tensors=[p.gpu.k_codes[:-1], p.gpu.k_exps, p.gpu.v_codes, p.gpu.v_exps])
