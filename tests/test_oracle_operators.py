"""CPU pins of the oracle's teacher records, distillation loss and draft verification: worked values,
differences of the loss against its gradient, and the distribution that verified drafts follow."""
import numpy as np
import pytest

import oracle


def test_top_logits_order():
    z = np.array([[1.0, 3.0, -np.inf, 3.0, np.nan, 2.0, -0.0, 0.0]])
    v, i, lse = oracle.top_logits(z, 8)
    assert i.tolist() == [[4, 1, 3, 5, 0, 6, 7, 2]]
    assert np.isnan(v[0, 0]) and np.isnan(lse[0])
    _, _, lse = oracle.top_logits(np.log([[1.0, 2.0, 5.0]]) * 0.5, 1, tau=0.5)
    assert abs(lse[0] - np.log(8.0)) < 1e-15


def test_distill_worked():
    # q = (1, 2, 5) / 8, record: token 2 with mass 1/2, token 0 with mass 1/4, 1/4 left out
    z = np.log([[1.0, 2.0, 5.0]])
    r = oracle.distill_loss(z, np.log([[0.5, 0.25]]), [[2, 0]], [0.0])
    want = 0.5 * np.log(0.5 / 0.625) + 0.25 * np.log(0.25 / 0.125) + 0.25 * np.log(0.25 / 0.25)
    assert abs(r["kl"][0] - want) < 1e-15
    assert np.allclose(r["dlogits"], [[0.125 - 0.25, 0.0, 0.625 - 0.5]], atol=1e-15)
    r = oracle.distill_loss(z, np.log([[0.5, 0.25]]), [[2, 0]])
    assert np.allclose(r["dlogits"], [[0.125 - 1 / 3, 0.25, 0.625 - 2 / 3]], atol=1e-15)


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("tau", [1.0, 0.7])
@pytest.mark.parametrize("twice", [False, True])
def test_distill_gradient_is_the_losses_slope(tail, tau, twice):
    rng = np.random.default_rng(3)
    z = rng.normal(0, 2, (2, 9))
    ids = np.array([[3, 1, 8, -1], [0, 4, 4 if twice else 5, 2]])
    values = rng.normal(0, 1, (2, 4))
    lse = np.array([3.0, 3.5]) if tail else None
    args = dict(mask=[1, 1], token_scale=[0.5, 2.0], tau=tau, loss_scale=1.5)
    g = oracle.distill_loss(z, values, ids, lse, **args)["dlogits"]
    h = 1e-5
    for t in range(2):
        for v in range(9):
            e = np.zeros_like(z)
            e[t, v] = h
            up, down = (oracle.distill_loss(z + s * e, values, ids, lse, **args)["loss"] for s in (1, -1))
            # central differences: h^2 f''' / 6 and rounding 1e-16 / h
            assert abs((up - down) / (2 * h) - g[t, v]) < 1e-8


@pytest.mark.parametrize("with_draft", [False, True])
def test_verified_tokens_are_the_policys(with_draft):
    """The first emitted token of many verified sequences follows p (3 sigma of the counts)."""
    rng = np.random.default_rng(11)
    V, B = 6, 20000
    p = rng.normal(0, 1, V)
    q = p + rng.normal(0, 1, V)
    pq = np.exp(q) / np.exp(q).sum()
    x = rng.choice(V, size=B, p=pq) if with_draft else np.full(B, int(np.argmax(q)))
    target = np.broadcast_to(p, (B, 2, V))
    draft = np.broadcast_to(q, (B, 1, V)) if with_draft else None
    _, tok, lp = oracle.verify_drafts(target, x[:, None], rng.random((B, 1)), rng.random(B), draft)
    want = np.exp(p) / np.exp(p).sum()
    got = np.bincount(tok[:, 0], minlength=V) / B
    assert (np.abs(got - want) < 4 * np.sqrt(want * (1 - want) / B)).all()
    assert np.allclose(np.exp(lp[:, 0]), want[tok[:, 0]])
