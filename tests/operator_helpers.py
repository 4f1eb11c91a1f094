"""Inputs and comparisons of the tests of top_logits, distill_loss_fwd_bwd and verify_drafts.

Tolerances, from the kernels' arithmetic (u: half a rounding step of a type, 2^-24 for float32 and
2^-8 for bf16):
  * log-sum-exps: a 32-bit exponential 2^(z L - n) is off by |z L - n| 2^-24 ln 2 (its argument's
    rounding) and 2^-22 (the exponential), and L itself by 2^-25; with |z / tau| <= 64 and the
    terms that matter within 32 log2 units of the maximum that stays below 32 * 2^-24 + 2^-22 +
    64 * 2^-25 = 4.1e-6 of the sum. LSE = 1e-5 * max(1, |lse|) adds the result's own rounding.
  * kl: sums of p (log p - log q) in 64 bits over a log q that is off by the same 4.1e-6, so
    KL = 1e-5 * max(1, |kl|).
  * dlogits: u |value| for the rounding, and GRAD = 2e-5 of the terms it is the difference of (the
    exponential of z L - lse2, |z L - lse2| <= 150 in the tests: 150 * 2^-24 * ln 2 = 6.2e-6, and
    the log-sum-exp's 4.1e-6); results below the type's normal range are flushed or rounded by up
    to 2^-126.
  * log-probs of verify_drafts: of accepted drafts, rounded once (u |lp|) from a row's log-sum-exp as
    above (LSE); of the drawn token, rounded once from 64-bit sums (1e-11).
"""
import numpy as np
import torch

from helpers import bits_of

DEV = "cuda:0"
LSE = KL = 1e-5
GRAD = 2e-5
U = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def rows(T, V, dtype, seed, sigma=3.0, ld=None, offset=0, lead=()):
    """[T, V] logits N(0, sigma^2) inside a buffer of row stride ld, `offset` entries in."""
    ld = V if ld is None else ld
    g = torch.Generator().manual_seed(seed)
    buf = torch.full((T * ld + offset + 64,), 77.0).to(dtype)
    z = (sigma * torch.randn(T, V, generator=g)).to(dtype)
    view = buf.as_strided((T, V), (ld, 1), offset)
    view.copy_(z)
    buf = buf.to(DEV)
    return buf.as_strided((T, V), (ld, 1), offset)


def near(got, want, tol, what):
    got, want = np.asarray(got, dtype=np.float64), np.asarray(want, dtype=np.float64)
    same = (np.isnan(got) & np.isnan(want)) | (got == want)
    with np.errstate(invalid="ignore"):
        bad = ~same & ~(np.abs(got - want) <= tol)
    assert not bad.any(), (f"{what}: {int(bad.sum())} of {bad.size} off, first at {np.argwhere(bad)[0]}: "
                           f"{got[bad][0]!r} against {want[bad][0]!r}")


def values_of(t):
    return bits_of(t)
