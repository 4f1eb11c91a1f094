"""DistillLoss where its gradient is asked for in other ways than one plain backward."""
import pytest
import torch
from torch.utils.checkpoint import checkpoint

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
    for reentrant in (True, False):                # a backward inside a backward is a plain one
        loss = checkpoint(lambda t: P.DistillLoss.apply(t, values, ids, lse, None, None, None)[0], leaf,
                          use_reentrant=reentrant)
        leaf.grad = None
        loss.backward()
        assert torch.equal(leaf.grad, want)
    loss = P.DistillLoss.apply(leaf, values, ids, lse, None, None, None)[0]
    us = torch.tensor([1.0, 3.0], device=DEV)
    (gb,) = torch.autograd.grad(loss, leaf, us, is_grads_batched=True)
    assert torch.equal(gb[0], want) and torch.equal(gb[1], 3.0 * want)


def ppo(x, **kw):
    g = torch.Generator().manual_seed(3)
    T, V = x.shape
    ids = torch.randint(0, V, (T,), generator=g).to(DEV)
    lp, adv = torch.full((T,), -5.0, device=DEV), torch.randn(T, generator=g).to(DEV)
    return P.DecoupledPPOLoss.apply(x, ids, lp, lp, adv, None, None, kw)[0]


def distill(x, **kw):
    values, ids, lse = record(rows(*x.shape, x.dtype, seed=5), 8, 6)
    return P.DistillLoss.apply(x, values, ids, lse, None, None, kw)[0]


@pytest.mark.parametrize("loss", [distill, ppo])
def test_buffers_of_the_callers(loss):
    """dlogits into a buffer that autograd does not own: two calls before the first one's backward, and
    logits that another node of the graph has saved, raise instead of giving the wrong gradient."""
    z, _ = student()
    leaf = z.clone().requires_grad_(True)
    (want,) = torch.autograd.grad(loss(leaf), leaf)
    buf = torch.empty(6, 208, device=DEV)
    d = buf[:, :200]
    first = loss(leaf, dlogits=d)
    (g,) = torch.autograd.grad(first, leaf, retain_graph=True)
    assert torch.equal(g, want)
    second = loss(leaf * 2.0, dlogits=d)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        torch.autograd.grad(first, leaf)
    torch.autograd.grad(second, leaf)
    # in place: fine where nothing else needs the logits, refused where something does
    w = torch.eye(200, device=DEV).requires_grad_(True)
    x = z @ w
    (gw,) = torch.autograd.grad(loss(x, dlogits=x.detach()), w)
    assert torch.allclose(gw, z.t() @ want, rtol=0, atol=1e-4)
    x = leaf.exp()
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        torch.autograd.grad(loss(x, dlogits=x), leaf)


@pytest.mark.parametrize("loss", [distill, ppo])
def test_a_forward_without_a_gradient(loss):
    z, _ = student()
    leaf = z.clone().requires_grad_(True)
    want = loss(leaf)
    got = loss(leaf, want_dlogits=False)
    assert got.item() == want.item()
    with pytest.raises(RuntimeError, match="want_dlogits=False"):
        got.backward()
    with torch.no_grad():
        assert loss(leaf, want_dlogits=False).item() == want.item()
