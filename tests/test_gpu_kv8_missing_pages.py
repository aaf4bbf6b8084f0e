"""Chunk attention of the 8-bit cache with page IDs outside the pool: nothing of any
page stands in for a missing one."""
import numpy as np
import pytest
import torch

from oracle import kv8 as ref
from paper_2609_17475_amd import jfkv
from tests.kv8_cases import Pair, check_lse, check_out, check_weights, i32, rows, wide
from tests.test_gpu_kv8 import decode, prefill

pytestmark = pytest.mark.gpu


# what the pool's pages hold that nobody wrote: NaN codes and 2^128; zeros; finite codes
# and 2^100; and a page of someone else's values, 2^12 times as large
@pytest.mark.parametrize("fill", [0xFF, 0x00, 0xE3, "others"])
@pytest.mark.parametrize("missing", [(0,), (2,), (5,), (0, 1, 4), (3, 4, 5), (0, 1, 2, 3, 4, 5)])
@pytest.mark.parametrize("d,hq,block,bf16,T", [(64, 4, 16, False, 300), (128, 4, 64, True, 300),
                                               (256, 6, 32, False, 70), (128, 2, 32, False, 3)])
def test_pages_that_nobody_wrote(fill, missing, d, hq, block, bf16, T):
    rng = np.random.default_rng(d + len(missing))
    n, hkv = 375, 2
    p = Pair(64, hkv, d, block, 9, bf16, fill=0xFF if fill == "others" else fill)
    table = np.array([3, 1, 5, 8, 7, 2], np.int32)   # (page 0 is not of this request)
    p.fill(rng, [n], table[None])
    if fill == "others":
        p.fill(rng, [64], np.array([[0]], np.int32), 4096.0)
    bad = table.copy()
    bad[list(missing)] = [9, -1, 1 << 30, -(1 << 31), 9, -5][:len(missing)]
    q = rows(rng, T, hq, d, bf16, 0.7)
    scale = d ** -0.5
    r = ref.attend(p.host, wide(q), bad, n, scale)
    for split in (False, True):
        out, lse = prefill(p, q, bad, n - T, scale, split)
        check_out(out, r, d, bf16, "split %s" % split)
        check_lse(lse, r, d, n)
    before = rng.random((hkv, n)).astype(np.float32)
    w = torch.from_numpy(before).cuda()
    jfkv.jf_kv8_attn_weights(p.gpu, q.cuda(), lse, i32(bad), n - T, scale, w)
    r["dots"] *= 2  # (the lse's own error beside the scores')
    check_weights(w.cpu().numpy(), before, r["weights"], r, d, n, T * hq // hkv)
    q1 = q[T - 2:].view(1, 2, hq, d)
    r = ref.attend(p.host, wide(q1[0]), bad, n, scale)
    check_out(decode(p, q1, bad[None], [n], scale)[0], r, d, bf16)


def test_missing_pages_of_a_long_prefix():
    """Several splits, some of which see only missing pages."""
    rng = np.random.default_rng(1)
    P, hkv, d, n = 256, 8, 128, 9000
    pages = -(-n // P)
    p = Pair(P, hkv, d, 64, pages + 1, fill=0xFF)
    table = np.arange(1, pages + 1, dtype=np.int32)
    p.fill(rng, [n], table[None])
    bad = table.copy()
    bad[:12], bad[20:23] = -1, pages + 1
    q = rows(rng, 3, 8, d, False)
    assert jfkv.jf_kv8_prefill_workspace_bytes(p.lay, 3, 8, n - 3) > 3 * 8 * (d + 4) * 4 * 12
    r = ref.attend(p.host, wide(q), bad, n, 0.08)
    for split in (False, True):
        out, lse = prefill(p, q, bad, n - 3, 0.08, split)
        check_out(out, r, d, False, "split %s" % split)
        check_lse(lse, r, d, n)
