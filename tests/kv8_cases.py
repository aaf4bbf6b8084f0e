"""Builders and error bounds shared by the tests of the 8-bit cache."""
from __future__ import annotations

import numpy as np
import torch

from oracle import kv8 as ref
from paper_2609_17475_amd import jfkv

STALE = 0xFF  # unwritten slots hold NaN codes and an exponent of 2^128


def dtype_of(bf16):
    return torch.bfloat16 if bf16 else torch.float16


def rows(rng, n, heads, d, bf16, spread=1.0):
    """Random rows as a CPU tensor of the type, with a few large channels."""
    x = rng.standard_normal((n, heads, d)) * spread
    x[:, :, rng.integers(0, d, 3)] *= 8.0
    return torch.from_numpy(x).to(dtype_of(bf16))


def wide(t):
    """A tensor's exact values in 64 bits."""
    return t.double().cpu().numpy()


def i32(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")


class Pair:
    """The same cache on the device and in the plain implementation."""

    def __init__(self, P=64, hkv=2, d=128, block=32, pages=8, bf16=False, fill=STALE):
        self.lay = jfkv.layout(P, hkv, d, block, pages)
        self.gpu = jfkv.KV8Pool(self.lay, fill=fill)
        self.host = ref.Cache(P, hkv, d, block, pages, fill=fill)
        self.bf16 = bf16

    def append(self, k, v, cu, start, tables, **kw):
        jfkv.jf_kv8_append(self.gpu, k.cuda(), v.cuda(), i32(cu), i32(start), i32(tables), **kw)
        self.host.append(wide(k), wide(v), cu, start, tables)

    def fill(self, rng, lens, tables, spread=1.0):
        """Rows 0 .. len - 1 of each request."""
        n = sum(lens)
        k, v = (rows(rng, n, self.lay.num_kv_heads, self.lay.head_dim, self.bf16, spread)
                for _ in range(2))
        self.append(k, v, np.cumsum([0] + list(lens)).tolist(), [0] * len(lens), tables)

    def differing(self):
        """Arrays that differ between the two, with the first place."""
        torch.cuda.synchronize()
        bad = []
        for name, want in zip(("k_codes", "k_exps", "v_codes", "v_exps"), self.host.pool_bytes()):
            got = getattr(self.gpu, name).cpu().numpy()
            if not np.array_equal(got, want):
                at = np.nonzero(got != want)[0]
                bad.append("%s: %d bytes, first at %d: %02x, wanted %02x" % (
                    name, at.size, at[0], got[at[0]], want[at[0]]))
        return bad


def tables_for(rng, P, lens, pages):
    """Shuffled pages for requests of these lengths, -1 padded; the pages left over."""
    need = [max(1, -(-n // P)) for n in lens]
    perm = rng.permutation(pages)
    t = np.full((len(lens), max(need)), -1, np.int32)
    at = 0
    for b, n in enumerate(need):
        t[b, :n] = perm[at:at + n]
        at += n
    return t, perm[at:]


def half_step(bf16):
    return 2.0 ** -8 if bf16 else 2.0 ** -11


def score_error(r, d):
    """Bound on the relative error of an unnormalised weight: d products summed
    in fp32 (any order), the factor, the subtraction of the maximum (both at most
    the scores' size, plus the exponents' window) and the exponential."""
    return (d + 8) * 2.0 ** -24 * r["dots"] + 20 * 2.0 ** -24 + 2.0 ** -22


def check_out(got, r, d, bf16, what=""):
    """An output against 64 bits.  Besides the weights' own error (twice: in the
    numerator and in the sum), a weight is rounded to fp16 (2^-11 of itself, and
    2^-25 of the largest weight where it is subnormal) and the output to its type."""
    got = got.double().cpu().numpy()
    tol = ((2.0 ** -11 + 2 * score_error(r, d) + 2.0 ** -18) * r["spread"] + 2.0 ** -25 * r["allv"]
           + half_step(bf16) * 1.01 * np.abs(r["out"]) + (0 if bf16 else 2.0 ** -25))
    err = np.abs(got - r["out"])
    assert np.all(np.isfinite(got)), what + ": not finite"
    at = np.unravel_index(np.argmax(err - tol), err.shape)
    assert np.all(err <= tol), "%s: off by %.3g at %s (got %g, want %g, allowed %.3g)" % (
        what, err[at], at, got[at], r["out"][at], tol[at])


def check_lse(got, r, d, n, what=""):
    got = got.double().cpu().numpy()
    none = np.isneginf(r["lse"])
    assert np.array_equal(np.isneginf(got), none), what
    tol = score_error(r, d) + n * 2.0 ** -24 + 2.0 ** -22 * (1 + np.abs(np.where(none, 0, r["lse"])))
    err = np.abs(np.where(none, 0, got) - np.where(none, 0, r["lse"]))
    assert np.all(err <= tol), "%s: lse off by %.3g" % (what, err.max())


def check_weights(got, before, added, r, d, n, terms, what=""):
    """Weights before + added: each of `terms` addends has the weights' error
    twice and the sum's n roundings; the additions round too."""
    want = before.astype(np.float64) + added
    if not want.size:
        return
    tol = added * (2 * score_error(r, d) + (n + terms + 8) * 2.0 ** -24) + 2.0 ** -23 * want + 1e-30
    err = np.abs(got.astype(np.float64) - want)
    at = np.unravel_index(np.argmax(err - tol), err.shape)
    assert np.all(err <= tol), "%s: weight off by %.3g at %s (got %g, want %g)" % (
        what, err[at], at, got[at], want[at])
