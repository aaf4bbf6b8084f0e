"""Attention calls of the 8-bit cache near the limits that include/jfkv.h states for
their inputs (bf16: fp16 does not reach them)."""
import numpy as np
import pytest
import torch

from oracle import kv8 as ref
from paper_2609_17475_amd import jfkv
from tests.kv8_cases import Pair, check_lse, check_out, check_weights, i32, rows, tables_for, wide
from tests.test_gpu_kv8 import decode, prefill

pytestmark = pytest.mark.gpu

# sizes of q, k, v as powers of two (rows reach about 2^5 times that), and the scale's
NEAR = {
    "values": (0, 0, 84, -3.5),           # |v| < 2^90
    "small_values": (0, 0, -100, -3.5),
    "queries": (80, 0, 0, -83.5),         # sum |q| < 2^90
    "keys": (-107, 101, 0, 3.0),          # |softmax_scale k| < 2^110
    "small_keys": (80, -112, 0, 29.0),
    "no_keys": (80, -130, 0, 0.0),        # (rounded to zero: every weight is the same)
    "no_scale": (80, 20, 0, -140.0),
}


@pytest.mark.parametrize("near", sorted(NEAR))
@pytest.mark.parametrize("d,hkv,hq,sq,n,splits", [(64, 2, 4, 1, 300, 64), (128, 1, 4, 1, 4100, 64),
                                                  (256, 1, 6, 3, 1700, 64), (128, 2, 8, 2, 1500, 1)])
def test_inputs_near_their_limits(near, d, hkv, hq, sq, n, splits):
    rng = np.random.default_rng(d + n)
    qs, ks, vs, s = NEAR[near]
    scale = 2.0 ** s
    p = Pair(64, hkv, d, 32, -(-n // 64) + 1, True)
    tables, _ = tables_for(rng, 64, [n], -(-n // 64) + 1)
    k, v = (rows(rng, n, hkv, d, True, 2.0 ** e) for e in (ks, vs))
    q = rows(rng, sq, hq, d, True, 2.0 ** qs)
    big = [float(x.double().abs().max()) for x in (k, v)]
    assert float(q.double().abs().sum(2).max()) < 2.0 ** 90
    assert big[0] * scale < 2.0 ** 110 and big[1] < 2.0 ** 90
    p.append(k, v, [0, n], [0], tables)
    assert not p.differing()
    r = ref.attend(p.host, wide(q), tables[0], n, scale)
    w = torch.zeros(1, hkv, tables.shape[1] * 64, device="cuda")
    out = decode(p, q.view(1, sq, hq, d), tables, [n], scale, splits, weights=w)
    check_out(out[0], r, d, True, "decode")
    check_weights(w[0].cpu().numpy()[:, :n], np.zeros((hkv, n)), r["weights"], r, d, n, sq * hq // hkv)
    for split in (False, True):
        out, lse = prefill(p, q, tables[0], n - sq, scale, split)
        check_out(out, r, d, True, "split %s" % split)
        check_lse(lse, r, d, n)
    w.zero_()
    jfkv.jf_kv8_attn_weights(p.gpu, q.cuda(), lse, i32(tables[0]), n - sq, scale, w[0])
    r["dots"] *= 2  # (the lse's own error beside the scores')
    check_weights(w[0].cpu().numpy()[:, :n], np.zeros((hkv, n)), r["weights"], r, d, n, sq * hq // hkv)
