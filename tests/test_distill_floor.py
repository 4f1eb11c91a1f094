"""The distillation gradient on both sides of the student's least tail mass, 2^-24: the loss's slope above it, the
stated formula below it. On the CPU for the oracle, on the GPU for the kernel."""
import numpy as np
import pytest
import torch

import oracle
from operator_helpers import DEV, GRAD, near

V, TAU = 30, 1.3
FLOOR = 2.0 ** -24


def case(tail_mass):
    """A student with `tail_mass` outside a record of three tokens that has 0.7 of the teacher's mass."""
    rng = np.random.default_rng(5)
    ids = np.array([[4, 17, 29]], dtype=np.int32)
    p = np.array([[0.4, 0.2, 0.1]])
    z = rng.normal(0, 1, (1, V))
    inside = np.zeros(V, dtype=bool)
    inside[ids[0]] = True
    e = np.exp(z[0] / TAU)
    z[0, inside] += TAU * (np.log(e[~inside].sum() / e[inside].sum()) + np.log(1 - tail_mass) - np.log(tail_mass))
    values = (TAU * np.log(p)).astype(np.float32)
    return z.astype(np.float32), values, ids, np.zeros(1, dtype=np.float32), inside


def slope(z, values, ids, lse):
    h, out = 1e-5, np.empty(V)
    zz = z.astype(np.float64)
    for v in range(V):
        e = np.zeros_like(zz)
        e[0, v] = h
        up, down = (oracle.distill_loss(zz + s * e, values, ids, lse, tau=TAU)["loss"] for s in (1, -1))
        out[v] = (up - down) / (2 * h)
    return out


def softmax(z):
    q = np.exp(z[0].astype(np.float64) / TAU - (z[0] / TAU).max())
    return q / q.sum()


def surrogate(z, values, ids, inside):
    """What the gradient has beside the loss's slope below the floor."""
    q = softmax(z)
    p = np.exp(values[0].astype(np.float64) / TAU)
    Pt = 1.0 - p.sum()
    return np.where(inside, q * Pt, -q * Pt * q[inside].sum() / FLOOR) / TAU


@pytest.mark.parametrize("tail_mass", [0.3, 2.0 ** -20, 2.0 ** -23.5, 2.0 ** -24.5, 2.0 ** -30, 1e-13])
def test_oracle(tail_mass):
    z, values, ids, lse, inside = case(tail_mass)
    assert (softmax(z)[~inside].sum() > FLOOR) == (tail_mass > FLOOR)
    g = oracle.distill_loss(z, values, ids, lse, tau=TAU)["dlogits"][0]
    more = surrogate(z, values, ids, inside) if tail_mass < FLOOR else 0.0
    # central differences: h^2 f''' / 6 and 1e-15 (the loss's size 5) / h
    assert np.abs(slope(z, values, ids, lse) + more - g).max() < 2e-9


def test_the_gradient_is_continuous_at_the_floor():
    (a, b) = (oracle.distill_loss(*case(m)[:4], tau=TAU)["dlogits"] for m in (FLOOR * 1.001, FLOOR * 0.999))
    assert np.abs(a - b).max() < 1e-3


@pytest.mark.gpu
@pytest.mark.parametrize("tail_mass", [0.3, 2.0 ** -20, 2.0 ** -23.5, 2.0 ** -24.5, 2.0 ** -30, 1e-13])
def test_kernel(tail_mass):
    import paper_2605_12070_amd as P
    z, values, ids, lse, inside = case(tail_mass)
    r = P.distill_loss_fwd_bwd(*(torch.from_numpy(t).to(DEV) for t in (z, values, ids, lse)), temperature=TAU)
    ref = oracle.distill_loss(z, values, ids, lse, tau=TAU)
    got = r.dlogits[0].cpu().double().numpy()
    near(got, ref["dlogits"][0], GRAD * ref["slack"][0] + 2.0 ** -24 * np.abs(ref["dlogits"][0]) + 2.0 ** -126, "dlogits")
    more = surrogate(z, values, ids, inside) if tail_mass < FLOOR else 0.0
    assert np.abs(slope(z, values, ids, lse) + more - got).max() < 2e-9 + 2e-5 * ref["slack"].max()
