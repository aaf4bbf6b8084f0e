"""Attention of the 8-bit cache over value blocks of zeros, whose exponent is the
least there is (-126), and over values next to the least that bf16 holds."""
import numpy as np
import pytest
import torch

from oracle import kv8 as ref
from paper_2609_17475_amd import jfkv
from tests.kv8_cases import Pair, check_lse, check_out, check_weights, i32, rows, tables_for, wide
from tests.test_gpu_kv8 import decode, evict, prefill

pytestmark = pytest.mark.gpu

ZERO = {
    "all": lambda t, n: t >= 0,
    "first": lambda t, n: t < 64,
    "first_half": lambda t, n: t < n // 2,
    "middle": lambda t, n: (t >= n // 3) & (t < 2 * n // 3),
    "last": lambda t, n: t >= n - n // 3,
    "every_other_block": lambda t, n: t // 16 % 2 == 0,
    "every_other_tile": lambda t, n: t // 64 % 2 == 1,
}


def cache(P, hkv, d, block, bf16, lens, where, size=1.0):
    """A cache whose values are zero where said, and the page tables."""
    rng = np.random.default_rng(d + len(lens) + len(where))
    pages = sum(-(-max(n, 1) // P) for n in lens) + 4
    p = Pair(P, hkv, d, block, pages, bf16)
    tables, rest = tables_for(rng, P, lens, pages)
    k, v = rows(rng, sum(lens), hkv, d, bf16), rows(rng, sum(lens), hkv, d, bf16, size)
    at = np.concatenate([ZERO[where](np.arange(n), n) for n in lens])
    v[torch.from_numpy(at)] = 0.0
    p.append(k, v, np.cumsum([0] + lens).tolist(), [0] * len(lens), tables)
    return rng, p, tables, rest


@pytest.mark.parametrize("P,hkv,hq,d,block,bf16,lens,sq,splits", [
    (64, 1, 1, 64, 16, False, [33], 1, 1),
    (64, 2, 8, 128, 16, True, [700, 31, 257], 1, 8),
    (256, 8, 8, 128, 64, False, [3000], 1, 64),       # splits joined by the last of them
    (128, 1, 6, 256, 32, False, [900, 40], 3, 64),    # two column sets
    (128, 1, 24, 64, 16, True, [800], 1, 1),          # and one split
    (128, 4, 24, 256, 64, True, [2000], 3, 64),       # joined by a launch of its own
])
@pytest.mark.parametrize("where", sorted(ZERO))
def test_decode_over_zero_values(P, hkv, hq, d, block, bf16, lens, sq, splits, where):
    rng, p, tables, _ = cache(P, hkv, d, block, bf16, lens, where)
    q = rows(rng, len(lens) * sq, hq, d, bf16, 0.7).view(len(lens), sq, hq, d)
    scale = d ** -0.5
    w = torch.zeros(len(lens), hkv, tables.shape[1] * P, device="cuda")
    out = decode(p, q, tables, lens, scale, splits, weights=w)
    for b, n in enumerate(lens):
        r = ref.attend(p.host, wide(q[b]), tables[b], n, scale)
        check_out(out[b], r, d, bf16, "request %d" % b)
        check_weights(w[b].cpu().numpy()[:, :n], np.zeros((hkv, n)), r["weights"], r, d, n,
                      sq * hq // hkv)


@pytest.mark.parametrize("P,hkv,hq,d,block,bf16,T,prefix", [
    (64, 1, 1, 64, 16, False, 1, 0),
    (64, 2, 6, 128, 16, True, 65, 0),
    (128, 2, 4, 256, 32, False, 50, 333),
    (64, 1, 7, 64, 32, False, 130, 61),
    (256, 8, 8, 64, 64, True, 3, 5000),               # several splits
    (256, 8, 8, 128, 128, False, 2, 4500),
])
@pytest.mark.parametrize("where", sorted(ZERO))
def test_prefill_over_zero_values(P, hkv, hq, d, block, bf16, T, prefix, where):
    n = T + prefix
    rng, p, tables, _ = cache(P, hkv, d, block, bf16, [n], where)
    q = rows(rng, T, hq, d, bf16, 0.7)
    r = ref.attend(p.host, wide(q), tables[0], n, d ** -0.5)
    for split in (False, True):
        out, lse = prefill(p, q, tables[0], prefix, d ** -0.5, split)
        check_out(out, r, d, bf16, "split %s" % split)
        check_lse(lse, r, d, n)


@pytest.mark.parametrize("size", [2.0 ** -117, 2.0 ** -122])
@pytest.mark.parametrize("d,block", [(64, 16), (128, 64), (256, 32)])
def test_values_next_to_the_least(d, block, size):
    n = 300
    rng, p, tables, _ = cache(64, 1, d, block, True, [n], "every_other_block", size)
    q = rows(rng, 2, 4, d, True).view(1, 2, 4, d)
    r = ref.attend(p.host, wide(q[0]), tables[0], n, d ** -0.5)
    # Outputs below 2^-126 are subnormal: seven bits of fraction leave bf16 a step of
    # 2^-133 there, whatever the output's size, so its rounding is off by up to 2^-134
    # besides the relative half step (the bound takes 2^-25 of allv).
    r["allv"] += 2.0 ** (25 - 134)
    check_out(decode(p, q, tables, [n], d ** -0.5)[0], r, d, True)
    check_out(prefill(p, q[0], tables[0], n - 2, d ** -0.5)[0], r, d, True)


def test_over_an_evicted_cache_with_a_page_missing():
    """Positions that eviction moved from no page are zeros, in K and in V."""
    rng, p, tables, rest = cache(64, 2, 128, 32, False, [250], "last")
    bad = tables.copy()
    bad[0, 0] = -1
    dst = rest[:2].astype(np.int32)[None]
    w = rng.random((1, 2, 256)).astype(np.float32)
    w[:, :, :64] += 1.0  # (they stay, as the first of those kept)
    evict(p, bad, [250], w, 128, 10, dst)
    q = rows(rng, 3, 8, 128, False).view(1, 3, 8, 128)
    r = ref.attend(p.host, wide(q[0]), dst[0], 128, 0.1)
    check_out(decode(p, q, dst, [128], 0.1)[0], r, 128, False)
    out, lse = prefill(p, q[0], dst[0], 125, 0.1)
    check_out(out, r, 128, False)
    check_lse(lse, r, 128, 128)
    weights = torch.zeros(2, 128, device="cuda")
    jfkv.jf_kv8_attn_weights(p.gpu, q[0].cuda(), lse, i32(dst[0]), 125, 0.1, weights)
    r["dots"] *= 2  # (the lse's own error beside the scores')
    check_weights(weights.cpu().numpy(), np.zeros((2, 128)), r["weights"], r, 128, 128, 12)
