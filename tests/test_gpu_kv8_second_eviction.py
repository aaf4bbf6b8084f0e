"""A session of the 8-bit cache that goes on after an eviction: the weights of what was
kept grow further and say what the next eviction keeps."""
import numpy as np
import pytest
import torch

from oracle import kv8 as ref
from tests.kv8_cases import Pair, check_out, check_weights, rows, wide
from tests.test_gpu_kv8 import decode, evict

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,hq,block,bf16", [(64, 4, 16, False), (128, 8, 32, True), (256, 6, 64, False)])
def test_weights_go_on_after_an_eviction(d, hq, block, bf16):
    rng = np.random.default_rng(d)
    P, hkv, keep, recent, scale = 64, 2, 90, 12, d ** -0.5
    p = Pair(P, hkv, d, block, 16, bf16)
    perm = rng.permutation(16).astype(np.int32)
    tables = [perm[:8].reshape(2, 4), perm[8:].reshape(2, 4)]
    lens = [230, 61]                     # (the second is shorter than what may stay)
    p.fill(rng, lens, tables[0])
    w = torch.from_numpy(rng.random((2, hkv, 4 * P)).astype(np.float32)).cuda()
    for turn in range(3):
        t, dst = tables[turn % 2], tables[1 - turn % 2]
        for step in range(8):
            k, v = (rows(rng, 2, hkv, d, bf16) for _ in range(2))
            p.append(k, v, [0, 1, 2], lens, t)
            lens = [n + 1 for n in lens]
            q = rows(rng, 2, hq, d, bf16, 0.7).view(2, 1, hq, d)
            before = w.cpu().numpy()
            out = decode(p, q, t, lens, scale, weights=w)
            for b, n in enumerate(lens):
                r = ref.attend(p.host, wide(q[b]), t[b], n, scale)
                check_out(out[b], r, d, bf16)
                check_weights(w[b, :, :n].cpu().numpy(), before[b, :, :n], r["weights"], r, d, n, hq // hkv)
        kept = evict(p, t, lens, w.cpu().numpy(), keep, recent, dst[:, :2])
        lens = [min(n, keep) for n in lens]
        # rows of the new tables' stride: what was kept, then positions that nothing saw yet
        fresh = torch.zeros_like(w)
        at = torch.from_numpy(kept).cuda().long()
        fresh[:, :, :keep] = torch.where(at >= 0, w.gather(2, at.clamp_min(0)), 0.0)
        w = fresh
