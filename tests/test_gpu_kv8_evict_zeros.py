"""Eviction that keeps only the zeros of blocks with large exponents: the signs of zeros
stay, whatever exponent their new block gets."""
import numpy as np
import pytest
import torch

from tests.kv8_cases import Pair, dtype_of, rows, tables_for
from tests.test_gpu_kv8 import evict

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,block", [(64, 16), (128, 64), (256, 32), (128, 128)])
@pytest.mark.parametrize("bf16,large,small", [(False, 2.0 ** 13, 0.0), (True, 2.0 ** 30, 0.0),
                                              (True, 2.0 ** 60, 2.0 ** -118)])
def test_kept_zeros_of_large_blocks(d, block, bf16, large, small):
    """small: what some of the kept rows hold instead of zeros."""
    rng = np.random.default_rng(d + block)
    n, keep = 380, 150
    p = Pair(128, 2, d, block, 8, bf16)
    tables, rest = tables_for(rng, 128, [n], 8)
    k, v = (rows(rng, n, 2, d, bf16) for _ in range(2))
    stay = np.sort(rng.permutation(n)[:keep])
    factor = np.full(n, large)
    factor[stay] = 0.0
    factor[stay[::5]] = small
    factor = torch.from_numpy(factor)[:, None, None]
    k, v = ((x.double() * factor).to(dtype_of(bf16)) for x in (k, v))  # (-1 * 0 = -0)
    p.append(k, v, [0, n], [0], tables)
    assert not p.differing()
    w = np.zeros((1, 2, 384), np.float32)
    w[:, :, stay] = 1.0
    assert np.array_equal(evict(p, tables, [n], w, keep, 0, rest[:2].astype(np.int32)[None])[0, 0], stay)
