"""Attention of requests that share prefixes, over the 8-bit cache, against its plain
implementation in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import kv8 as ref
from paper_2609_17475_amd import jfkv
from tests.kv8_cases import Pair, check_lse, check_out, dtype_of, i32, rows, wide

pytestmark = pytest.mark.gpu


class Batch:
    """Requests in groups: group g's first shared[g] positions lie in its first request's
    pages; the other tables hold nothing for them (`stale`), and their slots in a page
    that begins before shared[g] are unwritten, but for the block that it lies in."""

    def __init__(self, rng, P, hkv, hq, d, block, bf16, sizes, shared, lens, sq, stale=-1, spread=1.0):
        self.sq, self.first = sq, np.cumsum([0] + list(sizes)).tolist()
        self.shared, self.lens, self.scale = list(shared), list(lens), d ** -0.5
        B = len(lens)
        group = np.repeat(np.arange(len(sizes)), sizes)
        lead = np.array(self.first)[group]
        starts = [0 if b == lead[b] else min(max(shared[group[b]], 0), max(lens[lead[b]], 0)) // block * block
                  for b in range(B)]
        pages_of = [range(s // P, -(-max(n, s) // P)) for s, n in zip(starts, lens)]
        pages = sum(len(r) for r in pages_of) + 2
        width = max([r.stop for r in pages_of] + [1])
        perm = iter(rng.permutation(pages))
        self.tables = np.full((B, width), stale, np.int32)
        for b, r in enumerate(pages_of):
            for i in r:
                self.tables[b, i] = next(perm)
        self.cut = [min(max(shared[g], 0), max(min(lens[lead[b]], width * P), 0)) if sizes[g] > 1 else 0
                    for b, g in enumerate(group)]
        self.lead = lead
        self.p = Pair(P, hkv, d, block, pages, bf16)
        counts = [max(n - s, 0) for s, n in zip(starts, lens)]
        n = sum(counts)
        if n:
            k, v = (rows(rng, n, hkv, d, bf16, spread) for _ in range(2))
            self.p.append(k, v, np.cumsum([0] + counts).tolist(), starts, self.tables)
        self.q = rows(rng, B * sq, hq, d, bf16, 0.7).view(B, sq, hq, d)

    def call(self, q=None, scale=None, ws=None, fill=0xFF, wide_table=False, **kw):
        """wide_table: as of requests that may grow (another kernel takes the groups then)."""
        q = (self.q if q is None else q).cuda()
        tables = self.tables
        if wide_table:
            P = self.p.lay.page_size
            tables = np.full((len(tables), 2 ** 25 // (q[..., 0].numel() * P) + 1), -1, np.int32)
            n = min(self.tables.shape[1], tables.shape[1])
            tables[:, :n] = self.tables[:, :n]
            assert n == self.tables.shape[1] or (self.tables[:, n:] < 0).all()
        lay = self.p.lay
        if ws is None:
            n = jfkv.jf_kv8_shared_workspace_bytes(lay, q.shape[0], len(self.shared), self.sq, q.shape[2])
            ws = torch.full((n,), fill, dtype=torch.uint8, device="cuda")
        out = torch.full_like(q, 7.0)
        lse = torch.full(q.shape[:3], 7.0, device="cuda")
        jfkv.jf_kv8_shared_attn(self.p.gpu, q, i32(tables), i32(self.lens), i32(self.first),
                                i32(self.shared), self.scale if scale is None else scale, ws, out,
                                lse=lse, **kw)
        return out, lse

    def want(self, b, scale=None):
        p, lead, cut = self.p.host, self.tables[self.lead[b]], self.cut[b]

        class Seen:  # the positions before `cut` through the first request's table
            hkv = p.hkv

            def values(self, which, table, n, h):
                x, ok = p.values(which, table, n, h)
                c = min(cut, n)
                if c > 0:
                    y, on = p.values(which, lead, c, h)
                    x, ok = x.copy(), ok.copy()
                    x[:c], ok[:c] = y, on
                return x, ok

        n = min(max(self.lens[b], 0), self.tables.shape[1] * self.p.lay.page_size)
        return ref.attend(Seen(), wide(self.q[b]), self.tables[b], n, self.scale if scale is None else scale)

    def check(self, out, lse, scale=None, only=None):
        d, bf16 = self.q.shape[3], self.q.dtype == torch.bfloat16
        for b in only if only is not None else range(len(self.lens)):
            r = self.want(b, scale)
            check_out(out[b], r, d, bf16, "request %d" % b)
            check_lse(lse[b], r, d, max(self.lens[b], 1), "request %d" % b)
            none = np.isneginf(r["lse"])
            assert not out[b].cpu().double().numpy()[none].any()


CASES = [  # P, hkv, hq, d, block, bf16, sizes, shared, lens, sq
    (64, 1, 1, 64, 16, False, [1], [0], [1], 1),
    (64, 1, 4, 64, 16, False, [2], [64], [65, 66], 1),
    (64, 2, 8, 128, 32, False, [3], [192], [200, 193, 330], 1),
    (64, 2, 8, 128, 32, True, [3, 1, 2], [100, 50, 129], [200, 150, 101, 70, 140, 131], 1),
    (128, 1, 6, 256, 64, True, [4], [300], [310, 301, 700, 303], 3),
    (256, 2, 2, 64, 128, False, [5], [511], [512, 513, 600, 515, 1030], 4),
    (64, 1, 7, 128, 16, False, [9], [333], [340 + 7 * i for i in range(9)], 2),
    (64, 4, 16, 64, 64, True, [20], [128], [129 + i for i in range(20)], 1),
    (64, 1, 20, 128, 16, False, [2, 2], [17, 64], [60, 90, 64, 65], 4),
    (64, 1, 5, 256, 16, False, [11], [200], [205 + i for i in range(11)], 1),
    (64, 3, 3, 64, 16, False, [40], [96], [97 + i for i in range(40)], 1),
    (64, 1, 33, 128, 32, True, [7], [640], [645 + 50 * i for i in range(7)], 3),
    (256, 1, 4, 128, 64, False, [70], [1024], [1025 + 3 * i for i in range(70)], 1),
    (256, 1, 12, 256, 64, False, [33], [1024], [1028 + 3 * i for i in range(33)], 2),
    (256, 2, 4, 64, 64, True, [130], [512], [513 + (i * 37) % 200 for i in range(130)], 2),
]


@pytest.mark.parametrize("P,hkv,hq,d,block,bf16,sizes,shared,lens,sq", CASES)
def test_shared(P, hkv, hq, d, block, bf16, sizes, shared, lens, sq):
    rng = np.random.default_rng(hq + d + len(lens))
    b = Batch(rng, P, hkv, hq, d, block, bf16, sizes, shared, lens, sq)
    out, lse = b.call()
    b.check(out, lse)
    again, lse2 = b.call(fill=0x55)  # what the workspace held does not matter
    assert torch.equal(out, again) and torch.equal(lse, lse2)
    no_lse = torch.empty_like(out)
    ws = torch.empty(jfkv.jf_kv8_shared_workspace_bytes(b.p.lay, len(lens), len(sizes), sq, hq),
                     dtype=torch.uint8, device="cuda")
    jfkv.jf_kv8_shared_attn(b.p.gpu, b.q.cuda(), i32(b.tables), i32(lens), i32(b.first), i32(shared),
                            b.scale, ws, no_lse)
    assert torch.equal(out, no_lse)


WIDE = [c for c in CASES if len(c[8]) * c[2] // c[1] * c[9] > 128] + [
    # columns of full tiles and of what is left over (16, 32, 33, 128, 129), several groups
    (64, 1, 4, 64, 16, False, [68, 1, 40], [300, 77, 65], [303 + i % 50 for i in range(109)], 1),
    (64, 2, 16, 128, 32, True, [36], [640], [643 + 5 * i for i in range(36)], 1),
    (64, 1, 3, 128, 64, False, [11, 32], [130, 64], [140 + 7 * i for i in range(43)], 1),
    (128, 1, 8, 64, 16, False, [16, 48], [256, 1000], [1001 + i for i in range(64)], 1),
    (256, 1, 43, 256, 128, True, [3, 1], [700, 0], [701, 900, 702, 90], 3),
    (64, 2, 6, 256, 16, False, [48], [200], [205 + 3 * i for i in range(48)], 3),
    (64, 1, 1, 128, 16, True, [129, 2], [90, 100], [91 + i for i in range(131)], 1),
]


@pytest.mark.parametrize("P,hkv,hq,d,block,bf16,sizes,shared,lens,sq", WIDE)
def test_wide_tables(P, hkv, hq, d, block, bf16, sizes, shared, lens, sq):
    rng = np.random.default_rng(hq + d + len(lens) + 1)
    b = Batch(rng, P, hkv, hq, d, block, bf16, sizes, shared, lens, sq)
    out, lse = b.call(wide_table=True)
    b.check(out, lse)
    again, lse2 = b.call(wide_table=True, fill=0x55)
    assert torch.equal(out, again) and torch.equal(lse, lse2)
    b.check(*b.call())


@pytest.mark.parametrize("d", [64, 128, 256])
def test_wide_tables_where_it_goes_wrong(d):
    """Short and empty requests, no requests' own positions, pages outside the pool, bounds that
    do not ascend, negative scales: with tiles."""
    rng = np.random.default_rng(d)
    lens = [400] + [int(x) for x in rng.integers(0, 700, 79)]
    lens[5:9] = [0, 399, 400, 401]
    b = Batch(rng, 64, 1, 4, d, 16, d == 128, [80], [400], lens, 1)
    b.check(*b.call(wide_table=True))
    b.check(*b.call(wide_table=True, scale=-0.2), scale=-0.2)
    c = Batch(rng, 64, 1, 4, d, 16, d == 128, [80], [256], [256] * 80, 1)
    c.check(*c.call(wide_table=True))
    c.tables[0, 2] = len(c.p.host.pool_bytes()[0])  # (beyond any page)
    c.check(*c.call(wide_table=True))
    b.first, b.cut = [0, 81], [0] * 80  # every request by itself
    b.tables[1:, :7] = b.tables[0, :7]
    b.lens = [min(n, 400) for n in b.lens]
    b.check(*b.call(wide_table=True))


@pytest.mark.parametrize("sq", [1, 3])
def test_lengths_on_either_side_of_the_shared_positions(sq):
    """Requests that end before, at and just behind them, or hold nothing; groups of one, of
    none, and whose shared positions are more than the first request has."""
    rng = np.random.default_rng(sq)
    sizes = [6, 0, 1, 3, 2, 2]
    shared = [130, 40, 500, 1000, -5, 70]
    lens = [135, 130, 131, 60, 1, 0, 77, 90, 200, 88, 30, 40, 0, 20]
    b = Batch(rng, 64, 2, 6, 64, 16, False, sizes, shared, lens, sq)
    b.check(*b.call())


def test_lengths_outside_the_table():
    rng = np.random.default_rng(3)
    b = Batch(rng, 64, 1, 2, 64, 16, False, [3], [100], [128, 128, 128], 1)
    b.lens = [5000, -7, 2 ** 31 - 1]
    b.cut = [100] * 3
    b.check(*b.call())


def test_bounds_that_do_not_ascend_mean_no_groups():
    rng = np.random.default_rng(4)
    b = Batch(rng, 64, 2, 4, 128, 32, False, [1] * 6, [0] * 6, [70, 200, 65, 300, 1, 130], 1)
    want = b.call()
    b.check(*want)
    b.shared = [64, 64, 64]
    for first in ([0, 4, 2, 6], [1, 2, 3, 6], [0, 2, 4, 5], [0, 2, 4, 7], [-1, 2, 4, 6], [0, 2 ** 30, 3, 6]):
        b.first = first
        b.check(*b.call())


def test_pages_outside_the_pool():
    rng = np.random.default_rng(5)
    b = Batch(rng, 64, 2, 4, 128, 32, True, [3], [256], [300, 400, 500], 2)
    b.tables[0, 1], b.tables[0, 3] = b.p.lay.num_pages, -3  # of the shared positions
    b.tables[1, 5], b.tables[2, 4] = 2 ** 31 - 1, -1        # of their own
    b.check(*b.call())
    b.tables[:] = -1
    out, lse = b.call()
    assert not out.any() and torch.isneginf(lse).all()


@pytest.mark.parametrize("scale", [0.3, -0.3, 0.0, 1e-30])
def test_scales(scale):
    rng = np.random.default_rng(6)
    b = Batch(rng, 64, 1, 2, 64, 16, False, [10], [150], [160 + i for i in range(10)], 1)
    b.check(*b.call(scale=scale), scale=scale)


@pytest.mark.parametrize("d,bf16", [(64, False), (128, True), (256, False)])
@pytest.mark.parametrize("count", [2, 5, 40])
def test_where_exponents_jump(d, bf16, count):
    """Blocks whose values differ by up to 2^24: no common reference holds them."""
    rng = np.random.default_rng(d + count)
    lens = [420 + 3 * i for i in range(count)]
    b = Batch(rng, 64, 1, 4, d, 16, bf16, [count], [400], lens, 1)
    n = 400
    size = np.exp2(rng.integers(-12, 13, n // 16)).repeat(16)[:, None, None]
    k = rows(rng, n, 1, d, bf16)
    v = (rows(rng, n, 1, d, False).double() * torch.from_numpy(size)).to(dtype_of(bf16))
    b.p.append(k, v, [0, n], [0], b.tables[:1])
    b.check(*b.call())
    b.check(*b.call(wide_table=True))
    v[:] = v.abs() + 1  # and a needle: all weight on a position whose values are the smallest
    v[100:104] = 2.0 ** -12
    k[100] = 8.0
    b.p.append(k, v, [0, n], [0], b.tables[:1])
    b.q[:] = 1.0
    b.check(*b.call())
    b.check(*b.call(wide_table=True))


def test_many_items():
    """More groups and requests than a block looks at together, most of them empty."""
    rng = np.random.default_rng(8)
    sizes = [1 if i % 3 else 2 for i in range(900)]
    B = sum(sizes)
    shared = [int(x) for x in rng.integers(0, 40, 900)]
    lens = [int(n) if rng.random() < 0.3 else 0 for n in rng.integers(0, 60, B)]
    b = Batch(rng, 64, 1, 1, 64, 16, False, sizes, shared, lens, 1)
    b.check(*b.call())
    b.check(*b.call(wide_table=True))
    sizes, shared = [B], [0]  # one group, nothing shared
    c = Batch(rng, 64, 1, 2, 64, 16, True, sizes, shared, lens, 1)
    c.check(*c.call())
    c.check(*c.call(wide_table=True))


def test_most_requests():
    """As many requests as a call may have, most of them empty, in groups of one and of three."""
    rng = np.random.default_rng(13)
    B = 65535
    lens = np.zeros(B, int)
    some = np.sort(rng.permutation(B)[:300])
    lens[some] = rng.integers(1, 50, 300)
    lens[-3:] = [20, 30, 17]
    sizes = [1, 3] * 16383 + [3]
    b = Batch(rng, 64, 1, 1, 64, 16, False, sizes, [16] * len(sizes), lens.tolist(), 1)
    empty = torch.from_numpy(lens == 0).cuda()
    for wide_table in (False, True):
        out, lse = b.call(wide_table=wide_table)
        b.check(out, lse, only=[0, 1] + some[::4].tolist() + [B - 3, B - 2, B - 1])
        assert not out[empty].any() and torch.isneginf(lse[empty]).all()
        assert torch.isfinite(out).all() and torch.isfinite(lse[~empty]).all()


def test_long_line():
    """A prefix that every block takes a piece of, and one long request beside it."""
    rng = np.random.default_rng(9)
    b = Batch(rng, 256, 1, 4, 128, 64, False, [3, 1], [30000, 0], [30100, 30001, 30040, 9000], 1)
    b.check(*b.call())


@pytest.mark.parametrize("hq,hkv,d,block,bf16,sq,count", [(8, 2, 128, 64, False, 1, 40), (6, 1, 256, 32, True, 3, 12),
                                                         (16, 2, 64, 16, False, 2, 30)])
def test_against_the_decode_that_reads_prefixes_for_each(hq, hkv, d, block, bf16, sq, count):
    """Forked page tables: the same positions through jf_kv8_decode_attn."""
    rng = np.random.default_rng(count)
    P, prefix = 256, 5120
    lens = [prefix + sq + int(x) for x in rng.integers(0, 700, count)]
    pool_pages = prefix // P + sum(-(-(n - prefix) // P) for n in lens) + 1
    pool = jfkv.PagePool(pool_pages, P, shuffle_seed=5)
    lead = pool.create()
    pool.reserve(lead, prefix)
    pool.set_length(lead, prefix)
    seqs = [pool.fork(lead, prefix) for _ in lens]
    for s, n in zip(seqs, lens):
        pool.reserve(s, n)
        pool.set_length(s, n)
    width = -(-max(lens) // P)
    tables, got = pool.export(seqs, width)
    tables = np.asarray(tables, np.int32).reshape(count, width)
    pair = Pair(P, hkv, d, block, pool_pages, bf16)
    lay, cache = pair.lay, pair.gpu
    for which, start, n in [(0, 0, prefix)] + [(b, prefix, m - prefix) for b, m in enumerate(lens)]:
        k, v = (rows(rng, n, hkv, d, bf16) for _ in range(2))
        pair.append(k, v, [0, n], [start], tables[which:which + 1])
    q = rows(rng, count * sq, hq, d, bf16, 0.7).view(count, sq, hq, d).cuda()
    a, b = torch.empty_like(q), torch.empty_like(q)
    ws = torch.zeros(jfkv.jf_kv8_decode_workspace_bytes(lay, count, sq, hq, 64), dtype=torch.uint8, device="cuda")
    jfkv.jf_kv8_decode_attn(cache, q, i32(tables), i32(lens), d ** -0.5, 64, ws, a)
    ws = torch.empty(jfkv.jf_kv8_shared_workspace_bytes(lay, count, 1, sq, hq), dtype=torch.uint8, device="cuda")
    jfkv.jf_kv8_shared_attn(cache, q, i32(tables), i32(lens), i32([0, count]), i32([prefix]), d ** -0.5, ws, b)
    for i in range(0, count, 5):
        r = ref.attend(pair.host, wide(q[i]), tables[i], lens[i], d ** -0.5)
        check_out(a[i], r, d, bf16, "for each, request %d" % i)
        check_out(b[i], r, d, bf16, "once, request %d" % i)


def test_two_streams_and_a_graph():
    """Two calls at once with workspaces of their own; a captured call replayed with other
    lengths, groups and queries."""
    rng = np.random.default_rng(11)
    b = Batch(rng, 64, 2, 8, 128, 16, False, [1] * 5, [0] * 5, [700, 300, 650, 64, 500], 1)
    b.tables[1:, :4] = b.tables[0, :4]  # 256 positions that all of them share
    n = jfkv.jf_kv8_shared_workspace_bytes(b.p.lay, 5, 2, 1, 8)
    q, out = b.q.cuda(), torch.empty_like(b.q, device="cuda")
    tables, lens, first, shared = i32(b.tables), i32(b.lens), i32([0, 3, 5]), i32([256, 64])
    w1, w2 = (torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda") for _ in range(2))
    lse = torch.empty(5, 1, 8, device="cuda")
    call = [b.p.gpu, q, tables, lens, first, shared, b.scale]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        jfkv.jf_kv8_shared_attn(*call, w1, out, lse=lse)
    side = torch.cuda.Stream()
    out2 = torch.empty_like(out)
    for turn in range(4):
        b.lens = [int(x) for x in rng.integers(260, 300, 5)] if turn else [700, 300, 650, 64, 500]
        b.lens[3] = 64 if turn % 2 else 0
        b.q = rows(rng, 5, 8, 128, False, 0.7).view(5, 1, 8, 128)
        q.copy_(b.q)
        lens.copy_(torch.tensor(b.lens, dtype=torch.int32))
        b.first, b.shared = ([0, 3, 5], [256, 0]) if turn < 2 else ([0, 1, 3], [77, 256])
        if turn == 3:
            b.first, b.shared = [0, 2, 5], [192, 1000]
        first.copy_(torch.tensor(b.first, dtype=torch.int32))
        shared.copy_(torch.tensor(b.shared, dtype=torch.int32))
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            jfkv.jf_kv8_shared_attn(*call, w2, out2)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, out2)
        valid = b.first[-1] == 5
        lead = np.repeat(b.first[:-1], np.diff(b.first)) if valid else np.arange(5)
        b.lead = lead
        b.cut = [0] * 5
        if valid:
            for g in range(2):
                if b.first[g + 1] - b.first[g] > 1:
                    for r in range(b.first[g], b.first[g + 1]):
                        b.cut[r] = min(b.shared[g], b.lens[b.first[g]])
        b.check(out, lse)


def test_pages_beyond_32_bits():
    rng = np.random.default_rng(12)
    P, hkv, d = 256, 8, 128
    pages = 17000  # 4.46e9 codes in each of K and V
    lay = jfkv.layout(P, hkv, d, 64, pages)
    cache = jfkv.KV8Pool(lay, fill=0xFF)
    small = jfkv.layout(P, hkv, d, 64, 8)
    near = jfkv.KV8Pool(small, fill=0xFF)
    far_t = np.array([[16999, 16385, 16990], [16999, 16385, 16700]], np.int32)
    near_t = np.array([[1, 5, 3], [1, 5, 7]], np.int32)
    k, v = (rows(rng, 1300, hkv, d, False).cuda() for _ in range(2))
    for pool, t in ((cache, far_t), (near, near_t)):
        jfkv.jf_kv8_append(pool, k, v, i32([0, 700, 888]), i32([0, 512]), i32(t))
    q = rows(rng, 2, 32, d, False, 0.7).view(2, 1, 32, d).cuda()
    got = []
    for pool, t in ((cache, far_t), (near, near_t)):
        ws = torch.empty(jfkv.jf_kv8_shared_workspace_bytes(pool.layout, 2, 1, 1, 32), dtype=torch.uint8, device="cuda")
        out = torch.empty_like(q)
        jfkv.jf_kv8_shared_attn(pool, q, i32(t), i32([700, 700]), i32([0, 2]), i32([512]), d ** -0.5, ws, out)
        got.append(out)
    assert torch.equal(*got)


def test_refusals_of_the_binding():
    rng = np.random.default_rng(13)
    b = Batch(rng, 64, 1, 2, 64, 16, False, [2], [64], [70, 80], 1)
    n = jfkv.jf_kv8_shared_workspace_bytes(b.p.lay, 2, 1, 1, 2)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    q, t, lens, first, shared = b.q.cuda(), i32(b.tables), i32(b.lens), i32(b.first), i32(b.shared)
    out = torch.empty_like(q)

    def call(pool=b.p.gpu, q=q, t=t, lens=lens, first=first, shared=shared, ws=ws, out=out, lse=None):
        jfkv.jf_kv8_shared_attn(pool, q, t, lens, first, shared, 0.1, ws, out, lse=lse)

    for change in (dict(q=q.float()), dict(q=q[0]), dict(q=q.cpu()), dict(out=out.bfloat16()),
                   dict(t=t[:1]), dict(lens=lens[:1]), dict(first=first[:1]), dict(shared=shared.long()),
                   dict(lse=torch.empty(2, 1, 3, device="cuda")), dict(out=out[:, :, :1])):
        with pytest.raises(ValueError):
            call(**change)
    with pytest.raises(jfkv.JfError):
        call(ws=ws[:-16])
    with pytest.raises(jfkv.JfError):  # more groups than requests
        call(first=i32([0, 1, 2, 2]), shared=i32([0, 0, 0]))
    call()
