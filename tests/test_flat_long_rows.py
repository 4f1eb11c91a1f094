"""Log-sum-exps of rows of up to 2^28 equal logits, whose sums of exponentials round to one side.

Bound on a log-sum-exp: 4.1e-6 of the sum for the exponentials (operator_helpers), 20 joins of partial sums
at 2^-24 each, a thread's own sum in 64 bits or over 64 chunks at 2^-24 (3.8e-6); the result's rounding on top.
"""
import math

import numpy as np
import pytest
import torch

import paper_2605_12070_amd as P
from operator_helpers import DEV, GRAD, U, near

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
SUM = 4.1e-6 + 20 * 2.0 ** -24 + 3.8e-6


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,V", [(2, 151936), (2, 262144), (1, 524288), (1, 1 << 24), (600, 1 << 20), (3, (1 << 26) - 5), (1, 1 << 28)])
@pytest.mark.parametrize("tau", [1.0, 0.7])
def test_flat_rows(dtype, T, V, tau):
    print(f"[case] flat {dtype} T={T} V={V} tau={tau}", flush=True)
    z = torch.full((1, V), 2.1, device=DEV).to(dtype).expand(T, V).contiguous()
    x = float(z[0, 0]) / tau
    lse = x + math.log(V)
    r = P.top_logits(z, 3, temperature=tau)
    assert r.ids.tolist() == [[0, 1, 2]] * T
    near(r.lse.cpu().numpy(), np.full(T, lse), SUM + 2.0 ** -24 * lse, "lse")
    # a record of two tokens with 3/4 of the teacher's mass
    ids = torch.tensor([[5, V - 1]], dtype=torch.int32, device=DEV).expand(T, 2).contiguous()
    p = torch.tensor([0.5, 0.25], dtype=torch.float64)
    values = (tau * torch.log(p)).float().to(DEV).expand(T, 2).contiguous()
    p = torch.exp(values[0].cpu().double() / tau)
    d = P.distill_loss_fwd_bwd(z, values, ids, torch.zeros(T, device=DEV), temperature=tau, scale_mode="const")
    Pt, Qt = 1.0 - float(p.sum()), 1.0 - 2.0 / V
    kl = float((p * (torch.log(p) + math.log(V))).sum()) + Pt * math.log(Pt / Qt)
    near(d.kl.cpu().numpy(), np.full(T, kl), SUM + 2.0 ** -24 * kl, "kl")
    f = (float(p.sum()) - Pt * (2.0 / V) / Qt) / V / tau
    got = d.dlogits[:, 6:V - 1]
    assert float((got.max() - f).abs()) <= (U[dtype] + GRAD) * f and float((got.min() - f).abs()) <= (U[dtype] + GRAD) * f
