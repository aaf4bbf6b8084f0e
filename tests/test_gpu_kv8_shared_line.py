"""Attention of requests that share prefixes where the groups' units are many, or their
items more than a block looks at together, so that units lie on one line that is cut
into pieces: tiles that begin and end inside a unit, and blocks with several of them."""
import numpy as np
import pytest
import torch

from paper_2609_17475_amd import jfkv
from tests.kv8_cases import i32, rows
from tests.test_gpu_kv8_shared import Batch

pytestmark = pytest.mark.gpu


def own(rng, n, lo=1, hi=20):
    return [int(x) for x in rng.integers(lo, hi, n)]


def run(b, only):
    # tables wide enough for a kernel of the groups' own
    columns, P = b.q[..., 0].numel(), b.p.lay.page_size
    grow = columns * b.tables.shape[1] * P <= 2 ** 25
    out, lse = b.call(wide_table=grow)
    b.check(out, lse, only=only)
    again, lse2 = b.call(wide_table=grow, fill=0x55)  # what the workspace held does not matter
    assert torch.equal(out, again) and torch.equal(lse, lse2)
    if grow:
        b.check(*b.call(), only=only)


@pytest.mark.parametrize("hkv,hq,d,bf16,alone,size,shared", [
    (8, 32, 128, False, 300, 64, 512),
    (8, 32, 128, True, 256, 64, 1024),
    (8, 32, 64, False, 300, 64, 512),
    (2, 8, 64, True, 420, 100, 1500),
    (1, 8, 128, False, 310, 33, 65),
    (4, 16, 256, False, 300, 40, 512),
])
def test_a_group_beside_requests_alone(hkv, hq, d, bf16, alone, size, shared):
    """A step of the widest tiles costs more than a piece need be long."""
    rng = np.random.default_rng(alone + shared)
    lens = own(rng, alone) + [shared + n for n in own(rng, size)]
    b = Batch(rng, 64, hkv, hq, d, 16, bf16, [1] * alone + [size], [0] * alone + [shared], lens, 1)
    run(b, [0, alone - 1] + list(range(alone, alone + size, 7)))


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("pairs,shared,more", [(17, 32, 128), (16, 32, 320), (30, 64, 1000)])
def test_a_group_beside_pairs(d, pairs, shared, more):
    rng = np.random.default_rng(d + pairs)
    sizes = [2] * pairs + [64]
    lens = [shared + n for n in own(rng, 2 * pairs)] + [more + n for n in own(rng, 64)]
    b = Batch(rng, 64, 8, 32, d, 32, d == 64, sizes, [shared] * pairs + [more], lens, 1)
    run(b, list(range(0, 2 * pairs, 5)) + list(range(2 * pairs, 2 * pairs + 64, 7)))


@pytest.mark.parametrize("hkv,gq,d,sq,sizes,shared", [
    # several units a block, among them tiles of one set and of two, and rows
    (32, 2, 64, 1, [300, 290, 3, 270, 20], [200, 130, 77, 65, 500]),
    (16, 4, 128, 1, [100, 70, 40, 80, 5, 60], [700, 300, 64, 129, 1000, 448]),
    (16, 2, 256, 2, [70, 33, 9, 48, 65, 40], [400, 257, 640, 64, 130, 200]),
    # units of many pieces
    (20, 2, 64, 4, [70, 66, 65, 64], [3000, 2000, 1000, 1500]),
])
def test_long_lines_of_tiles(hkv, gq, d, sq, sizes, shared):
    rng = np.random.default_rng(hkv + d)
    lens = [s + sq + n for s, size in zip(shared, sizes) for n in own(rng, size)]
    lens[1], lens[sizes[0] + 1] = 0, shared[1] - 3  # and requests that end before their group's positions
    b = Batch(rng, 64, hkv, hkv * gq, d, 64, d == 128, sizes, shared, lens, sq)
    ends = np.cumsum([0] + sizes).tolist()
    run(b, sorted({i for lo, hi in zip(ends, ends[1:]) for i in (lo, lo + 1, (lo + hi) // 2, hi - 1)}))


@pytest.mark.parametrize("d,bf16", [(128, False), (256, True)])
def test_captured_with_other_groups(d, bf16):
    """A captured call over wide tables, replayed with groups, lengths and queries that put
    its units on a line or not, with the same call on another stream beside it."""
    rng = np.random.default_rng(d)
    B, G, hkv, hq = 100, 40, 8, 32
    lens = [int(x) for x in rng.integers(260, 400, B)]
    b = Batch(rng, 64, hkv, hq, d, 16, bf16, [1] * B, [0] * B, lens, 1)
    b.tables[1:, :4] = b.tables[0, :4]  # 256 positions that all of them share
    tables = np.full((B, 2 ** 25 // (B * hq * 64) + 1), -1, np.int32)
    tables[:, :b.tables.shape[1]] = b.tables
    b.tables = tables
    groups = [
        ([0] + [B] * G, [256] + [0] * (G - 1)),                                   # one of all
        (list(range(0, 2 * G, 2)) + [B], [int(x) for x in rng.integers(1, 257, G)]),  # pairs, and one of 22
        (list(range(G)) + [B], [0] * (G - 1) + [200]),                            # alone, and one of 61
        ([0, 50] + [B] * (G - 1), [130, 256] + [7] * (G - 2)),
    ]
    n = jfkv.jf_kv8_shared_workspace_bytes(b.p.lay, B, G, 1, hq)
    w1, w2 = (torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda") for _ in range(2))
    q = b.q.cuda()
    out, out2, lse = torch.empty_like(q), torch.empty_like(q), torch.empty(B, 1, hq, device="cuda")
    lens_d, first, shared = i32(lens), i32(groups[0][0]), i32(groups[0][1])
    call = [b.p.gpu, q, i32(tables), lens_d, first, shared, b.scale]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        jfkv.jf_kv8_shared_attn(*call, w1, out, lse=lse)
    side = torch.cuda.Stream()
    for turn, (bounds, most) in enumerate(groups + groups[:2]):
        b.first, b.shared = bounds, most
        b.lens = [0 if x < 10 else int(rng.integers(257, m + 1)) for x, m in zip(rng.integers(0, 100, B), lens)]
        for lo in bounds[:-1]:
            if lo < B:
                b.lens[lo] = lens[lo]  # (whose table is read)
        b.lead = np.repeat(bounds[:-1], np.diff(bounds))
        wide = np.repeat(np.where(np.diff(bounds) > 1, most, 0), np.diff(bounds))
        b.cut = [int(x) for x in wide]
        b.q = rows(rng, B, hq, d, bf16, 0.7).view(B, 1, hq, d)
        for to, new in ((q, b.q), (lens_d, i32(b.lens)), (first, i32(bounds)), (shared, i32(most))):
            to.copy_(new)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            jfkv.jf_kv8_shared_attn(*call, w2, out2)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, out2)
        b.check(out, lse, only=sorted(set(range(turn, B, 9)) | {0, B - 1}))
