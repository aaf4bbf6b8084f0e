"""The write of rotated keys where the angles outgrow an XCD's cache and a unit's heads are
started together: bit for bit a rotation and an append."""
import numpy as np
import pytest
import torch

from paper_2609_17475_amd import jfkv
from tests.kv8_cases import dtype_of, i32
from tests.test_gpu_rope import make_table

pytestmark = pytest.mark.gpu
CODES = ("k_codes", "k_exps", "v_codes", "v_exps")


def randn(gen, n, heads, d, bf16):
    return (torch.randn((n, heads, d), generator=gen, device="cuda") * 3).to(dtype_of(bf16))


@pytest.mark.parametrize("P,hkv,gq,d,block,rot,pairs,bf16,lens,prefix,skip", [
    # angles of 4 MB, of one row more, and more (130, 130 and 627 units)
    (256, 1, 4, 128, 64, 128, False, False, [8192], 0, 0),
    (256, 1, 4, 128, 64, 128, False, False, [8193], 0, 0),
    (64, 3, 2, 128, 16, 128, True, True, [10001], 37, 0),
    # several requests, odd lengths, rows in the middle of a block, tokens of no request
    (256, 3, 1, 128, 64, 128, False, True, [3001, 1, 0, 64, 7003, 12], 51, 5),
    (128, 1, 7, 256, 128, 256, True, False, [1, 2111, 999, 1500, 63], 100, 3),
    (64, 2, 3, 256, 32, 64, False, False, [9000, 8999], 7, 0),
    (64, 8, 1, 64, 16, 64, True, False, [5] * 400 + [15001], 3, 17),
])
def test_rope_append_is_rotate_then_append(P, hkv, gq, d, block, rot, pairs, bf16, lens, prefix, skip):
    rng = np.random.default_rng(len(lens) + d + rot)
    gen = torch.Generator(device="cuda").manual_seed(d + rot)
    n, hq, B = sum(lens) + 2 * skip, hkv * gq, len(lens)
    need = [-(-(m + prefix) // P) for m in lens]
    perm, at = rng.permutation(sum(need) + 2).tolist(), 0
    tables = np.full((B, max(need)), -1, np.int32)
    for b, m in enumerate(need):
        tables[b, :m] = perm[at:at + m]
        at += m
    tables[0, need[0] // 2] = [-1, 10 ** 9][skip % 2] if need[0] > 2 else tables[0, need[0] // 2]  # rows without a page
    lay = jfkv.layout(P, hkv, d, block, sum(need) + 2)
    one, two = (jfkv.KV8Pool(lay, fill=0xA5) for _ in range(2))
    if prefix:
        m = prefix * B
        k, v = (randn(gen, m, hkv, d, bf16) for _ in range(2))
        for pool in (one, two):
            jfkv.jf_kv8_append(pool, k, v, i32(np.arange(B + 1) * prefix), i32([0] * B), i32(tables))
    cu, start, tab = i32(skip + np.cumsum([0] + list(lens))), i32([prefix] * B), i32(tables)
    table = make_table(rng, n + 3, rot)
    assert (n * rot * 4 > 4 << 20) == (n != 8192)
    x = torch.cat([randn(gen, n, h, d, bf16) for h in (hq, hkv, hkv)], 1)  # one projection's rows
    q, k, v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:].contiguous()
    for rows, apart in ((None, False), (i32(rng.integers(0, n + 3, n)), True)):
        rope = jfkv.Rope(table, rows=rows, pairs=pairs)
        turned_q = torch.empty((n, hq, d), dtype=x.dtype, device="cuda")
        turned_k = torch.empty((n, hkv, d), dtype=x.dtype, device="cuda")
        jfkv.jf_rope_rotate(rope, q, turned_q, k, turned_k)
        jfkv.jf_kv8_append(two, turned_k, v, cu, start, tab)
        if apart:  # without queries
            jfkv.jf_kv8_rope_append(one, rope, k, v, cu, start, tab)
        else:
            out = torch.full((n + 1, hq, d), 3.0, dtype=x.dtype, device="cuda")
            jfkv.jf_kv8_rope_append(one, rope, k, v, cu, start, tab, q=q, q_out=out[:n])
            assert torch.equal(out[:n].view(torch.int16), turned_q.view(torch.int16))
            assert (out[n] == 3.0).all()
        for name in CODES:
            assert torch.equal(getattr(one, name), getattr(two, name)), name
