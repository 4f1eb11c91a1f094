"""verify_drafts against the 64-bit oracle."""
import numpy as np
import pytest
import torch

import oracle
import paper_2605_12070_amd as P
from operator_helpers import DEV, LSE, near, values_of

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def inputs(B, D, V, dtype, seed, drafts="logits", noise=0.7, sigma=3.0):
    g = torch.Generator().manual_seed(seed)
    z = (sigma * torch.randn(B, D + 1, V, generator=g)).to(dtype)
    q = (z[:, :D].float() + noise * torch.randn(B, D, V, generator=g)).to(dtype)
    x = q.double()
    if drafts == "logits":
        x = x - torch.log(-torch.log(torch.rand(B, D, V, generator=g, dtype=torch.float64).clamp_min(1e-300)))
    ids = x.argmax(2) if D else torch.empty(B, 0, dtype=torch.int64)
    u, un = torch.rand(B, D, generator=g), torch.rand(B, generator=g)
    q = q.to(DEV) if drafts == "logits" else None
    return z.to(DEV), ids.to(DEV), u.to(DEV), un.to(DEV), q


def check(z, ids, u, un, q=None, n=None, tau=1.0):
    r = P.verify_drafts(z, ids, u, un, q, n, temperature=tau)
    torch.cuda.synchronize()
    B, D1, V = z.shape
    f = lambda t: None if t is None else values_of(t.reshape(-1, V)).reshape(t.shape)  # noqa: E731
    acc, tok, lp = oracle.verify_drafts(f(z), ids.cpu().numpy(), u.cpu().numpy(), un.cpu().numpy(), f(q),
                                        None if n is None else n.cpu().numpy(), tau)
    assert np.array_equal(r.accepted.cpu().numpy(), acc), "accepted"
    assert np.array_equal(r.tokens.cpu().numpy(), tok), "tokens"
    drawn = np.arange(D1)[None] == acc[:, None]
    tol = np.where(drawn, 1e-11, LSE) + 2.0 ** -24 * np.abs(np.nan_to_num(lp))
    near(r.logp.cpu().numpy(), lp, tol, "logp")
    return r


@pytest.mark.parametrize("drafts", ["logits", "tokens"])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("B,D,V", [
    (1, 0, 5), (1, 1, 1), (2, 3, 2), (4, 2, 7), (3, 4, 100), (40, 5, 257), (5, 1, 1000), (6, 8, 1023), (2, 70, 300),
    (3, 3, 5000), (33, 2, 4099), (2, 4, 32000), (3, 2, 50257), (2, 3, 151936), (1, 2, 262144), (300, 2, 600),
])
def test_random_batches(dtype, B, D, V, drafts):
    print(f"[case] verify {dtype} B={B} D={D} V={V} {drafts}", flush=True)
    z, ids, u, un, q = inputs(B, D, V, dtype, seed=B + D + V, drafts=drafts)
    check(z, ids, u, un, q, tau=1.0 if V % 2 else 0.8)
    n = torch.randint(-1, D + 2, (B,), generator=torch.Generator().manual_seed(V), dtype=torch.int32).to(DEV)
    check(z, ids, u, un, q, n)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("offset,q_offset", [(0, 0), (1, 1), (3, 4), (2, 7)])
def test_strides_and_offsets(dtype, offset, q_offset):
    print(f"[case] verify {dtype} offset={offset} q_offset={q_offset}", flush=True)
    B, D, V = 4, 3, 1501
    z, ids, u, un, q = inputs(B, D, V, dtype, seed=7)
    zs = torch.zeros(B * 5 * 1507 + 64, dtype=dtype, device=DEV).as_strided((B, D + 1, V), (5 * 1507, 1507, 1), offset)
    qs = torch.zeros(B * 4 * 1510 + 64, dtype=dtype, device=DEV).as_strided((B, D, V), (4 * 1510, 1510, 1), q_offset)
    zs.copy_(z)
    qs.copy_(q)
    check(zs, ids, u, un, qs)
    # positions outermost in memory
    check(z.transpose(0, 1).contiguous().transpose(0, 1), ids, u, un, q)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("V", [1, 3, 4, 5, 7, 8, 9, 11, 15, 16, 17, 23])
def test_rows_around_one_chunk_at_every_offset(dtype, V):
    """Rows that hold no whole 16-byte chunk at their offset, the draft's rows at an allocation's start."""
    print(f"[case] verify chunk {dtype} V={V}", flush=True)
    B, D = 3, 2
    z, ids, u, un, q = inputs(B, D, V, dtype, seed=V)
    for offset in range(8):
        buf = torch.full((B * (D + 1) * V + 8,), 30.0, device=DEV).to(dtype)
        zz = buf[offset:offset + z.numel()].view(z.shape)
        zz.copy_(z)
        check(zz, ids, u, un, q.clone())
        check(zz, ids, u, un)


@pytest.mark.parametrize("drafts", ["logits", "tokens"])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("B,D,V,offset,shift", [(6, 3, 40, 0, 0.0), (5, 4, 1003, 1, 20.0), (4, 20, 5001, 3, -900.0),
                                                (3, 3, 50257, 0, 5000.0), (2, 3, 151936, 2, 0.0)])
def test_decisions_next_to_their_border(dtype, drafts, B, D, V, offset, shift):
    """Random numbers within a float's step of p / q: the 32-bit statistics cannot tell."""
    print(f"[case] verify border {dtype} {drafts} B={B} D={D} V={V}", flush=True)
    z, ids, u, un, q = inputs(B, D, V, dtype, seed=V + B, drafts=drafts, sigma=2.0)
    z = (z.float() + shift).to(dtype)
    buf = torch.zeros(z.numel() + 8, dtype=dtype, device=DEV)
    zz = buf[offset:offset + z.numel()].view(z.shape)
    zz.copy_(z)
    f = lambda t, i: np.take_along_axis(np.apply_along_axis(oracle.dppo_oracle.log_softmax_row, 2, values_of(  # noqa: E731
        t.reshape(-1, V)).reshape(t.shape)[:, :D]), i, 2)[:, :, 0]
    i = ids.cpu().numpy()[:, :, None]
    ratio = np.exp(f(z, i) - (f(q, i) if q is not None else 0.0))
    x = np.minimum(ratio, 1.0).astype(np.float32)
    steps = np.random.default_rng(V).integers(-1, 2, x.shape)
    x = np.where(steps > 0, np.nextafter(x, np.float32(2)), np.where(steps < 0, np.nextafter(x, np.float32(0)), x))
    margin = np.abs(x.astype(np.float64) / ratio - 1.0)
    # The inputs: decidable by sums of exponentials good to 4.5e-12 over two rows (9e-12), not in 32 bits.
    assert margin.min() > 2e-11 and (margin < 2e-7).any()
    check(zz, ids, torch.from_numpy(x).to(DEV), un, q)


@pytest.mark.parametrize("drafts", ["logits", "tokens"])
def test_ends_of_the_random_numbers(drafts):
    """u of 0 and just below 1 (and 1, which is outside the range), drafts equal to the policy, drafts
    the policy rules out."""
    B, D, V = 12, 3, 900
    z, ids, u, un, q = inputs(B, D, V, F32, seed=3, drafts=drafts)
    one = float(np.nextafter(np.float32(1), np.float32(0)))
    un[:4] = torch.tensor([0.0, one, 1.0, 0.5], device=DEV)
    u[0] = 0.0
    u[1] = one
    z[2, 0, int(ids[2, 0])] = -float("inf")
    u[2, 0] = 0.0
    if q is not None:
        q[3] = z[3, :D]
        q[4] = z[4, :D]
        u[4] = 1.0                      # rejects a draft that p equals: drawn from p itself
    z[5, :, 10:] = -float("inf")
    z[6, :, :890] = torch.finfo(F32).min
    z[7, 0] = -30.0
    z[7, 0, 899] = 30.0
    z[8] = torch.finfo(F32).min          # a mask that leaves nothing: even odds
    check(z, ids, u, un, q)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_flat_rows(dtype):
    """A thousand equal weights: every boundary of the running sum counts."""
    B, D, V = 64, 1, 1000
    z = torch.zeros(B, D + 1, V, dtype=dtype, device=DEV)
    ids = torch.randint(0, V, (B, D), generator=torch.Generator().manual_seed(1)).to(DEV)
    u = torch.rand(B, D, generator=torch.Generator().manual_seed(2)).to(DEV)
    # halfway between the boundaries
    un = ((torch.arange(B) * 15 + 0.5) / V).float().to(DEV)
    check(z, ids, u, un)
    q = torch.zeros(B, D, V, dtype=dtype, device=DEV)
    q[:, :, ::2] = 1.0
    check(z, ids, u, un, q)


def test_data_errors_end_a_sequence():
    B, D, V = 8, 3, 400
    z, ids, u, un, q = inputs(B, D, V, BF, seed=5)
    q[:] = z[:, :D]                      # accepted unless something is wrong
    ids[0, 1] = V
    ids[1, 0] = -1
    z[2, 2, 7] = float("nan")
    z[3, 0] = -float("inf")
    z[4, 3, 9] = float("inf")
    q[5, 1, 3] = float("nan")
    ids[6, 2] = -5
    n = torch.tensor([3, 3, 3, 3, 3, 3, 2, 3], dtype=torch.int32, device=DEV)
    r = check(z, ids, u, un, q, n)
    assert r.accepted.cpu().tolist() == [1, 0, 2, 0, 3, 1, 2, 3]


def test_empty_batch():
    r = P.verify_drafts(torch.empty(0, 3, 50, device=DEV), torch.empty(0, 2, dtype=torch.int64, device=DEV),
                        torch.empty(0, 2, device=DEV), torch.empty(0, device=DEV))
    assert r.tokens.shape == (0, 3)


def test_another_stream_and_the_same_bits_again():
    z, ids, u, un, q = inputs(30, 4, 9001, BF, seed=8)
    a = check(z, ids, u, un, q)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        b = P.verify_drafts(z, ids, u, un, q)
    s.synchronize()
    assert torch.equal(a.tokens, b.tokens) and torch.equal(a.logp, b.logp) and torch.equal(a.accepted, b.accepted)
