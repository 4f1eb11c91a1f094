"""top_logits, distill_loss_fwd_bwd and verify_drafts where a stretch of the vocabulary is masked with a finite
value: threads and parts that see nothing but the mask before, after or instead of ordinary logits."""
import numpy as np
import pytest
import torch

import oracle
import paper_2605_12070_amd as P
from operator_helpers import DEV, LSE, near, rows, values_of
from test_distill import compare, record
from test_verify import check, inputs

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
MASKS = [-1e5, -1e9, -2e9, -1e10, -1e20, -1e30, "lowest"]


def value(mask, dtype):
    return torch.finfo(dtype).min if mask == "lowest" else mask


def stretches(V):
    """Masked [from, to) of rows: the ends, the middle, all but a few at an end or inside."""
    return [(0, V // 2), (V // 2, V), (V // 3, V - V // 3), (0, V - 5), (5, V), (0, V - V // 9), (V // 9, V), (9, 9)]


def masked(V, dtype, mask, seed, T=8):
    z = rows(T, V, dtype, seed=seed).contiguous()
    for t, (a, b) in enumerate(stretches(V)):
        z[t, a:b] = value(mask, dtype)
    return z


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("tau", [0.7, 1.0, 2.0])
@pytest.mark.parametrize("V,T", [(1500, 300), (9001, 8), (9001, 2100), (50257, 8), (151936, 8)])
def test_top_logits(dtype, tau, V, T):
    for mask in MASKS:
        print(f"[case] mask top {dtype} tau={tau} {mask} V={V} T={T}", flush=True)
        z = masked(V, dtype, mask, V, T)
        r = P.top_logits(z, 40, temperature=tau)
        values, ids, lse = oracle.top_logits(values_of(z[:8]), 40, tau)
        assert np.array_equal(r.ids[:8].cpu().numpy(), ids) and np.array_equal(r.values[:8].cpu().double().numpy(), values)
        assert np.isfinite(lse).all()
        near(r.lse[:8].cpu().numpy(), lse, LSE * np.maximum(1, np.abs(lse)), "lse")


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("tail,tau", [(False, 1.0), (True, 2.0), (True, 0.7)])
@pytest.mark.parametrize("V", [600, 9001, 40000, 110000, 170001])
def test_distill(dtype, tau, V, tail):
    k = 6
    for mask in MASKS:
        print(f"[case] mask distill {dtype} tau={tau} {mask} tail={tail} V={V}", flush=True)
        z = masked(V, dtype, mask, V)
        values, ids, lse = record(z, k, 5, tau, short=False)
        # the record among what is left (a masked token in it has a divergence of the mask's size)
        for t, (a, b) in enumerate(stretches(V)):
            free = [v for v in list(range(0, a))[:k] + list(range(b, V))[-k:]][:k]
            ids[t, :len(free)] = torch.tensor(free, dtype=torch.int32, device=DEV)
            ids[t, len(free):] = -1
        r = P.distill_loss_fwd_bwd(z, values, ids, lse if tail else None, temperature=tau)
        ref = compare(r, z, values, ids, lse if tail else None, tau=tau)
        assert np.isfinite(ref["kl"]).all() and np.isfinite(ref["dlogits"]).all()


@pytest.mark.parametrize("drafts", ["logits", "tokens"])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("tau", [0.7, 1.0, 2.0])
@pytest.mark.parametrize("V", [1200, 40000])
def test_verify(dtype, tau, V, drafts):
    B, D = 8, 2
    for mask in MASKS:
        print(f"[case] mask verify {dtype} tau={tau} {mask} {drafts} V={V}", flush=True)
        z, ids, u, un, q = inputs(B, D, V, dtype, seed=V, drafts=drafts)
        for b, (lo, hi) in enumerate(stretches(V)):
            z[b, :, lo:hi] = value(mask, dtype)
            if q is not None and b % 3:
                q[b, :, lo:hi] = value(mask, dtype)
            if b % 2:
                ids[b] = lo - 1 if lo else hi
                u[b] *= 0.5
        ids.clamp_(0, V - 1)
        r = check(z, ids, u, un, q, tau=tau)
        assert bool((r.tokens[torch.arange(B, device=DEV), r.accepted.long()] >= 0).all())
