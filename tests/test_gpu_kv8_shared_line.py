"""Attention of requests that share prefixes where the groups' units are many, or their
items more than a block looks at together, so that units lie on one line that is cut
into pieces: tiles that begin and end inside a unit, and blocks with several of them."""
import numpy as np
import pytest
import torch

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
