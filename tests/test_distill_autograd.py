"""DistillLoss where its gradient is asked for in other ways than one plain backward."""
import pytest
import torch

import paper_2605_12070_amd as P
from operator_helpers import DEV, rows
from test_distill import record

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def student(dtype=F32, T=6, V=200):
    z = rows(T, V, dtype, seed=5).contiguous()
    return z, record(z, 8, 6)


@pytest.mark.filterwarnings("ignore:Using backward")
def test_second_derivatives_are_refused():
    """They were formed without the logits' part: a gradient penalty came out without its gradient."""
    z, (values, ids, lse) = student()
    leaf = z.clone().requires_grad_(True)
    want = P.distill_loss_fwd_bwd(z, values, ids, lse).dlogits
    for x in (leaf, leaf * 1.0):
        loss = P.DistillLoss.apply(x, values, ids, lse, None, None, None)[0]
        with pytest.raises(RuntimeError, match="second derivatives"):
            torch.autograd.grad(loss, leaf, create_graph=True)
    loss = P.DistillLoss.apply(leaf, values, ids, lse, None, None, None)[0]
    with pytest.raises(RuntimeError, match="second derivatives"):
        loss.backward(create_graph=True)
    # the same graph's plain and batched gradients
    loss = P.DistillLoss.apply(leaf, values, ids, lse, None, None, None)[0]
    (g,) = torch.autograd.grad(loss, leaf, retain_graph=True)
    assert torch.equal(g, want)
    us = torch.tensor([1.0, 3.0], device=DEV)
    (gb,) = torch.autograd.grad(loss, leaf, us, is_grads_batched=True)
    assert torch.equal(gb[0], want) and torch.equal(gb[1], 3.0 * want)
