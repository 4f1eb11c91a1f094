"""The loss stage where a stretch of the vocabulary is masked with a finite value: threads, chunks and shards
that hold nothing but the mask. The masked entries have no weight and no gradient, whatever the value.

Against float64 on the GPU. With logp_mu = logp_ref = the row's own log-prob the ratios are 1 up to the
log-prob's error (2e-5, helpers.TIGHT), the advantages 1 and the scale constant: dlogits = softmax - onehot,
bf16 entries to 2^-8 + 2^-11 of their value (helpers), 1e-4 for the ratio, 2^-22 for fp16's subnormals.
"""
import pytest
import torch

import paper_2605_12070_amd as P
from helpers import TIGHT

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32
MASKS = [-1e4, -5e7, -1e8, -1e9, -2e9, -1e10, -1e20, -1e30, "lowest"]


def stretches(V):
    return [(0, V // 2), (V // 2, V), (V // 3, V - V // 3), (5, V), (0, V - 5), (0, V - V // 9), (V // 9, V), (9, 9)]


def masked(V, dtype, mask, offset=0):
    g = torch.Generator().manual_seed(V)
    T = len(stretches(V))
    z = torch.empty(T * V + offset, device=DEV, dtype=dtype)[offset:].view(T, V)
    z.copy_(3 * torch.randn(T, V, generator=g))
    ids = torch.empty(T, dtype=torch.int64)
    for t, (a, b) in enumerate(stretches(V)):
        z[t, a:b] = torch.finfo(dtype).min if mask == "lowest" else mask
        ids[t] = a - 1 if a else min(b, V - 1)
    return z, ids.to(DEV)


def off(got, want, tol):
    return bool(((got.double() - want).abs() <= tol).all())      # False for NaN


@pytest.mark.parametrize("policy", ["auto", "stream"])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("V,offset", [(200, 0), (1501, 0), (1504, 3), (9000, 0), (32000, 0), (50257, 1), (98304, 0),
                                      (110001, 0), (151936, 0), (170001, 0), (300000, 2)])
def test_loss_stage(dtype, V, offset, policy):
    P.set_path_policy(policy)
    try:
        for mask in MASKS:
            print(f"[case] loss mask {dtype} V={V} offset={offset} {policy} {mask}", flush=True)
            z, ids = masked(V, dtype, mask, offset)
            T = z.shape[0]
            zz = z.double()
            lse = torch.logsumexp(zz, 1)
            lp = zz.gather(1, ids[:, None])[:, 0] - lse
            got, got_lse = P.logprob_fwd(z, ids, with_lse=True)
            assert off(got, lp, TIGHT * lp.abs().clamp_min(1)) and off(got_lse, lse, TIGHT * lse.abs().clamp_min(1)), mask
            ver = torch.zeros(T, dtype=torch.int32, device=DEV)
            assert off(P.logprob_fwd_versioned([z, z], ver, ids), lp, TIGHT * lp.abs().clamp_min(1)), mask
            r = P.decoupled_ppo_loss_fwd_bwd(z, ids, got, got, torch.ones(T, device=DEV), scale_mode="const")
            assert off(r.logp, lp, TIGHT * lp.abs().clamp_min(1)), mask
            want = torch.exp(zz - lse[:, None])
            want[torch.arange(T, device=DEV), ids] -= 1.0
            step = 2.0 ** -8 + 2.0 ** -11 if dtype == BF else 0.0
            assert off(r.dlogits, want, (step + 1e-4) * want.abs() + 2.0 ** -22), mask
    finally:
        P.set_path_policy("auto")


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("V", [3000, 40004])
def test_shards(dtype, V):
    """Columns in four shards, of which some are masked as a whole."""
    for mask in MASKS:
        print(f"[case] shard mask {dtype} V={V} {mask}", flush=True)
        z, ids = masked(V, dtype, mask)
        T, n = z.shape[0], V // 4
        zz = z.double()
        lse = torch.logsumexp(zz, 1)
        lp = zz.gather(1, ids[:, None])[:, 0] - lse
        parts = [z[:, s * n:(s + 1) * n] for s in range(4)]
        stats = [P.vocab_shard_stats(p, ids, s * n, V) for s, p in enumerate(parts)]
        got_lse = P.vocab_shard_combine(torch.stack([s[0] for s in stats]).contiguous())
        assert off(got_lse, lse, TIGHT * lse.abs().clamp_min(1)), mask
        mine = torch.stack([s[1] for s in stats]).sum(0)         # z[y] of the shard that has it
        assert off(mine, zz.gather(1, ids[:, None])[:, 0], 0.0)
