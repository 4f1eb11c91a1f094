"""verify_drafts with a sample_u at the ends of its range: the draw next to stretches of the vocabulary without
weight, which are longer than the cells that weights are summed over (64 chunks of 16 bytes)."""
import numpy as np
import pytest
import torch

import paper_2605_12070_amd as P
from operator_helpers import DEV
from test_verify import check, inputs

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
ONE = float(np.nextafter(np.float32(1), np.float32(0)))


@pytest.mark.parametrize("drafts", ["logits", "tokens"])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("mask", [-float("inf"), -1e10, -3000.0])
@pytest.mark.parametrize("V", [4001, 20000])
def test_ends_of_the_range_beside_masked_stretches(dtype, drafts, mask, V):
    """Leading, trailing and inner stretches that p and q both rule out, over sequences enough for both
    signs of what the statistics leave to the cells' sums."""
    print(f"[case] empty cells {dtype} {drafts} {mask} V={V}", flush=True)
    B, D = 64, 1
    z, ids, u, un, q = inputs(B, D, V, dtype, seed=V, drafts=drafts)
    a = V // 3
    for lo, hi, rows in ((0, a, slice(0, 48)), (V - a, V, slice(16, 64)), (a + 300, V - a - 9, slice(32, 64))):
        z[rows, :, lo:hi] = mask
        if q is not None:
            q[rows, :, lo:hi] = mask
    if q is not None:
        ids = (q[:, :, a:a + 300].float() - z[:, :D, a:a + 300].float()).argmax(2) + a    # q well above p: rejected
    else:
        ids = torch.full_like(ids, a + 7)
    u.fill_(ONE)
    u[::8] = 0.0                                   # some accepted: the draw is from p then
    un[0::4], un[1::4], un[2::4] = 0.0, 1.0, ONE
    r = check(z, ids, u, un, q)
    drawn = r.tokens[torch.arange(B, device=DEV), r.accepted.long()]
    assert bool((drawn >= 0).all()) and set(r.accepted.tolist()) == {0, 1}


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("lead", [True, False])
def test_weights_at_the_flush(dtype, lead):
    """A stretch of weights just under 1e-280 each, which count as 0 however many there are."""
    print(f"[case] weights at the flush {dtype} lead={lead}", flush=True)
    B, V, n = 8, 6000, 2500
    z = torch.full((B, 1, V), -30.0, device=DEV).to(dtype)
    z[:, :, 3000] = 2.0
    at = slice(0, n) if lead else slice(V - n, V)
    # p = e^(z - 2) (3000 weights of e^-32 do not show): 5e-281 at z = -643.46, e^-0.6 to 1 of it after rounding
    z[:, :, at] = -643.5
    assert 1e-281 < float(np.exp(float(z[0, 0, 0 if lead else V - 1]) - 2.0)) < 1e-280
    un = torch.tensor([0.0, 1.0, ONE, 0.5] * 2, device=DEV)
    none = torch.empty(B, 0, device=DEV)
    r = P.verify_drafts(z, none.long(), none, un)
    zz = z.clone()
    zz[:, :, at] = -float("inf")
    want = P.verify_drafts(zz, none.long(), none, un)
    first, last = (n, V - 1) if lead else (0, V - n - 1)
    assert want.tokens[:, 0].tolist() == [first, last, 3000, 3000] * 2
    assert torch.equal(r.tokens, want.tokens) and torch.equal(r.logp, want.logp)
