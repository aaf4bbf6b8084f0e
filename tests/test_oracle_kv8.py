"""The plain implementation of the 8-bit cache against independent facts (CPU)."""
import numpy as np
import pytest
import torch

from oracle import kv8 as ref


def test_code_values_are_e4m3():
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(t, ref.VALUES, equal_nan=True)


def test_encode_is_the_nearest_code_ties_to_even():
    fine = [c for c in range(256) if c & 127 != 127]
    assert np.array_equal(ref.encode(ref.VALUES[fine]), np.array(fine, np.uint8))
    mid = (ref.VALUES[:126] + ref.VALUES[1:127]) / 2
    got = ref.encode(mid)
    assert np.all(got % 2 == 0) and np.all(np.abs(got - np.arange(126.0) - 0.5) == 0.5)
    assert np.array_equal(ref.encode(np.nextafter(mid, 0)), np.arange(126))
    assert np.array_equal(ref.encode(np.nextafter(mid, 1e9)), np.arange(1, 127))
    x = np.random.default_rng(0).standard_normal(20000) * 100
    x = np.float32(x[np.abs(x) <= 448])
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(ref.encode(x), want)


@pytest.mark.parametrize("amax", [2.0 ** -24, 1.0, 447.9, 448.0, 448.1, 65504.0, 3.38e38, 1e-40])
def test_exponent_is_the_least(amax):
    e = ref.exponent(amax)
    assert amax <= 448 * 2.0 ** e and (e == -126 or amax > 448 * 2.0 ** (e - 1))


def test_append_row_by_row_reads_back_within_half_a_step():
    rng = np.random.default_rng(1)
    c = ref.Cache(64, 1, 64, 16, 2)
    k, v = rng.standard_normal((2, 70, 1, 64)) * np.exp(rng.uniform(-3, 3, (2, 70, 1, 1)))
    table = [[1, 0]]
    for i in range(70):
        c.append(k[i:i + 1], v[i:i + 1], [0, 1], [i], table)
    whole = ref.Cache(64, 1, 64, 16, 2)
    whole.append(k, v, [0, 70], [0], table)
    assert all(np.array_equal(a, b) for a, b in zip(c.exps, whole.exps))
    for which, x in ((0, k), (1, v)):
        for cache in (c, whole):
            got, ok = cache.values(which, table[0], 70, 0)
            top = 2.0 ** (cache.exps[which][[1, 0]].reshape(-1)[np.arange(70) // 16].astype(float) - 127)
            # half a step of 3 mantissa bits; subnormal codes (steps of 2^-9) may have
            # been rounded once per growth of their block's exponent
            tol = np.abs(x[:, 0]) * 2.0 ** -4 + 2 * 2.0 ** -10 * top[:, None]
            assert ok.all() and np.all(np.abs(got - x[:, 0]) <= tol)


def test_layout_of_value_codes():
    c = ref.Cache(64, 2, 128, 16, 3)
    c.codes[1][:] = np.random.default_rng(2).integers(0, 255, c.codes[1].shape, np.uint8)
    flat = c.pool_bytes()[2]
    for page, h, t, dim in ((2, 1, 63, 127), (0, 0, 21, 70), (1, 1, 5, 3)):
        at = (page * 2 + h) * 64 * 128 + t // 16 * 16 * 128 + dim // 64 * 1024 \
            + t % 16 // 4 * 256 + dim % 64 // 4 * 16 + dim % 4 * 4 + t % 4
        assert flat[at] == c.codes[1][page, h, t, dim]


def test_attention_against_torch_and_shared_sums():
    rng = np.random.default_rng(3)
    c = ref.Cache(64, 2, 64, 32, 4)
    k, v = rng.standard_normal((2, 100, 2, 64))
    c.append(k, v, [0, 100], [0], [[3, 1]])
    q = rng.standard_normal((5, 6, 64))
    r = ref.attend(c, q, [3, 1], 100, 0.125)
    kk, vv = (np.stack([c.values(i, [3, 1], 100, h)[0] for h in range(2)]).repeat(3, 0) for i in range(2))
    mask = torch.ones(5, 100).tril(95).bool()
    want = torch.nn.functional.scaled_dot_product_attention(
        torch.from_numpy(q).transpose(0, 1), torch.from_numpy(kk), torch.from_numpy(vv),
        attn_mask=mask, scale=0.125).transpose(0, 1).numpy()
    assert np.abs(r["out"] - want).max() < 1e-12
    assert np.allclose(r["weights"].sum(1), 15.0)  # 5 rows, 3 heads each


def test_eviction_keeps_order_ties_and_nan():
    w = np.array([1.0, 5.0, 1.0, np.inf, 0.0, np.nan, 1.0, -0.0, 9.0, 9.0], np.float32)
    assert ref.pick(w, 10, 4, 1) == [3, 5, 8, 9]
    assert ref.pick(w, 10, 6, 2) == [0, 1, 3, 5, 8, 9]
    assert ref.pick(w, 10, 10, 0) == list(range(10))
    assert ref.pick(w, 3, 5, 4) == [0, 1, 2]
    assert ref.pick(np.zeros(6, np.float32), 6, 2, 0) == [0, 1]
    assert ref.pick(np.array([0.0, -0.0, -1.0, -0.0]), 4, 2, 0) == [0, 1]
