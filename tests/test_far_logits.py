"""top_logits and distill_loss_fwd_bwd on rows far from zero: a mask of a finite value that leaves nothing,
large offsets, temperatures that make ordinary logits large. Where the differences between a row's
logits are what counts, a rounded product with log2(e) / temperature has none of them left."""
import numpy as np
import pytest
import torch

import oracle
import paper_2605_12070_amd as P
from operator_helpers import DEV, LSE, near, rows, values_of
from test_distill import compare, record

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
TAUS = [0.5, 0.7, 1.0, 2.0, 4.0]


def far_rows(V, dtype, seed, T=10):
    """Ordinary rows, and rows of one far value, of one and its neighbours, and of one and -inf."""
    low = torch.finfo(dtype).min
    z = rows(T, V, dtype, seed=seed).contiguous()
    z[0].fill_(low)
    z[1].fill_(-1e9)
    z[2].fill_(-1e10)
    z[3].fill_(-1e30)
    z[4].fill_(3e12)
    z[5].fill_(low)
    z[5, ::3] = -float("inf")
    # neighbours of a far value: the larger ones have all of the softmax
    z[6].fill_(-7e9)
    ints = z.view(torch.int16 if dtype == BF else torch.int32)
    ints[6, ::2] += 1
    z[7].fill_(5e9)
    ints[7, 1::5] += 1
    z[8, 3:] = 2e11
    return z


def lse_near(r, z, tau):
    want = oracle.top_logits(values_of(z), 1, tau)[2]
    with np.errstate(over="ignore"):
        want = want.astype(np.float32)          # -inf where the value is past float32's range
    near(r.lse.cpu().numpy(), want, LSE * np.maximum(1, np.abs(np.nan_to_num(want))), "lse")


# a wave per row, a workgroup per row, rows in parts and their join
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("V,T", [(1, 10), (7, 300), (1001, 300), (5003, 2100), (5003, 10), (50257, 10), (262147, 10)])
def test_top_logits(dtype, V, T):
    z = far_rows(max(V, 10), dtype, V, T)[:, :V]
    k = min(V, 20)
    for tau in TAUS:
        print(f"[case] far top {dtype} tau={tau} V={V} T={T}", flush=True)
        r = P.top_logits(z, k, temperature=tau)
        values, ids, _ = oracle.top_logits(values_of(z[:10]), k, tau)
        assert np.array_equal(r.ids[:10].cpu().numpy(), ids)
        assert np.array_equal(r.values[:10].cpu().double().numpy(), values)
        lse_near(r, z, tau)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("V,T", [(90, 10), (90, 700), (2001, 700), (9001, 600), (40003, 10), (40003, 520), (70001, 10),
                                 (140001, 10), (170001, 10), (330001, 10), (90, 20000), (3001, 9000), (130001, 600),
                                 (170001, 520)])
def test_distill(dtype, tail, V, T):
    """Every shape's rows, in and out of place, several to a workgroup; a record with an empty, a doubled and a far value."""
    tau = TAUS[(V + tail) % 5]
    print(f"[case] far distill {dtype} tail={tail} V={V} T={T} tau={tau}", flush=True)
    k = 12
    z = far_rows(V, dtype, V, 10)
    flat = rows(10, V, dtype, seed=V).contiguous()
    values, ids, lse = record(flat, k, 5, tau, short=False)
    ids[0, 3] = -1
    ids[2, 7] = ids[2, 2]
    values[3] = values[3] - 1e6                   # a teacher far from zero; with the tail its own lse
    lse[3] = lse[3] - 1e6 / tau
    at = torch.arange(T, device=DEV) % 10
    mask = torch.ones(T, dtype=torch.uint8, device=DEV)
    mask[9::10] = 0
    many = [t[at].contiguous() for t in (z, values, ids, lse)]
    r = P.distill_loss_fwd_bwd(many[0], many[1], many[2], many[3] if tail else None, mask, temperature=tau)
    torch.cuda.synchronize()
    assert int(r.stats[0]) == T - T // 10
    near(r.flags.cpu().numpy(), mask.cpu().numpy(), 0, "flags")
    n = int(r.stats[0])
    # a batch's rows repeat the first ten, which the oracle knows
    first = P.DistillResult(r.loss, r.kl[:10], r.flags[:10], torch.tensor([9, 0, 0, 0, 0]), r.dlogits[:10])
    ref = oracle.distill_loss(values_of(z), values.cpu().numpy(), ids.cpu().numpy(),
                              lse.cpu().double().numpy() if tail else None, mask[:10].cpu().numpy(), None, tau,
                              "const", 1.0 / n)
    first.loss = torch.tensor([ref["loss"]])
    compare(first, z, values, ids, lse if tail else None, mask[:10], tau=tau, scale_mode="const", loss_scale=1.0 / n)
    assert bool((r.kl.view(-1, 10) == r.kl[:10]).all())
    for some in r.dlogits.view(-1, 10, V).split(100):
        assert bool((some == r.dlogits[:10]).all())
    want = sum(ref["kl"][i % 10] for i in range(T) if i % 10 != 9) / n
    near(r.loss.cpu().numpy(), [want], 2e-5 * max(1.0, np.abs(ref["kl"]).max()), "loss")
    again = P.distill_loss_fwd_bwd(many[0], many[1], many[2], many[3] if tail else None, mask, temperature=tau,
                                   dlogits=many[0])
    assert torch.equal(again.dlogits, r.dlogits) and torch.equal(again.kl, r.kl)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("tail", [False, True])
def test_far_tokens_of_the_record(dtype, tail):
    """The record's own tokens far above or below the rest, and a record beside a far rest."""
    print(f"[case] far record {dtype} tail={tail}", flush=True)
    V, k = 3001, 6
    z = rows(6, V, dtype, seed=3).contiguous()
    values, ids, lse = record(z, k, 5, short=False)
    at = ids.long()
    z[0, at[0, 1]] = 1e10
    z[1, at[1]] = 4e9
    z[2, at[2, :5]] = -1e10
    keep = z[3, at[3]].clone()
    z[3].fill_(-3e10)
    z[3, at[3]] = keep
    z[4, [v for v in range(10) if v not in ids[4].tolist()][0]] = 6e9
    r = P.distill_loss_fwd_bwd(z, values, ids, lse if tail else None)
    torch.cuda.synchronize()
    compare(r, z, values, ids, lse if tail else None)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_smallest_temperature(dtype):
    """tau = 1e-6: the largest logit takes the softmax, at logits of a few hundred as at few."""
    print(f"[case] far temperature {dtype}", flush=True)
    z = rows(8, 4003, dtype, seed=2, sigma=3.0).contiguous()
    z[1] += 900.0
    z[2] -= 5000.0
    z[3].fill_(2000.0)
    r = P.top_logits(z, 9, temperature=1e-6)
    lse_near(r, z, 1e-6)
    values, ids, lse = record(z, 5, 3, 1e-6, short=False)
    d = P.distill_loss_fwd_bwd(z, values, ids, None, temperature=1e-6, loss_scale=1e-6)
    torch.cuda.synchronize()
    compare(d, z, values, ids, None, tau=1e-6, loss_scale=1e-6)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("V", [77, 9001, 150001])
def test_far_rows_with_nothing_in_the_record(dtype, tail, V):
    """Empty records, and records of tokens that the row rules out."""
    print(f"[case] far empty record {dtype} tail={tail} V={V}", flush=True)
    k = 5
    z = far_rows(V, dtype, V)
    values, ids, lse = record(rows(10, V, dtype, seed=4).contiguous(), k, 5, short=False)
    ids[:8] = -1
    z[8, ids[8].long()] = -float("inf")
    lse[8] = float("inf")                          # p = 0: the tail has all of the teacher's mass
    r = P.distill_loss_fwd_bwd(z, values, ids, lse if tail else None)
    torch.cuda.synchronize()
    ref = oracle.distill_loss(values_of(z), values.cpu().numpy(), ids.cpu().numpy(),
                              lse.cpu().double().numpy() if tail else None)
    fine = np.isfinite(ref["kl"])
    assert fine[:8].all() and (fine[8] or not tail)
    near(r.kl.cpu().numpy(), ref["kl"], 1e-5 * np.maximum(1, np.abs(np.nan_to_num(ref["kl"]))), "kl")
    got, tol = values_of(r.dlogits), 2.0 ** -8 * np.abs(ref["dlogits"]) + 2e-5 * ref["slack"] + 2.0 ** -126
    near(got[fine], ref["dlogits"][fine], tol[fine], "dlogits")


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("V", [1, 3, 77, 9001])
def test_rows_without_a_softmax_and_without_a_record(dtype, V):
    """NaN, +inf and -inf alone stay visible in a loss that is the tail's alone."""
    print(f"[case] no softmax {dtype} V={V}", flush=True)
    z = rows(8, V, dtype, seed=V).contiguous()
    z[0] = -float("inf")
    z[1, V // 2] = float("nan")
    z[2, V - 1] = float("inf")
    z[4] = -float("inf")
    z[5, 0] = float("nan")
    z[6, V // 3] = float("inf")
    ids = torch.full((8, 2), -1, dtype=torch.int32, device=DEV)
    ids[4:, 0] = 0
    values = torch.full((8, 2), -float("inf"), device=DEV)      # p = 0
    lse = torch.zeros(8, device=DEV)
    r = P.distill_loss_fwd_bwd(z, values, ids, lse)
    ref = oracle.distill_loss(values_of(z), values.cpu().numpy(), ids.cpu().numpy(), lse.cpu().double().numpy())
    assert np.isnan(ref["kl"]).tolist() == [True, True, True, False] * 2
    near(r.kl.cpu().numpy(), ref["kl"], 1e-5 * np.maximum(1, np.abs(np.nan_to_num(ref["kl"]))), "kl")
    assert torch.isnan(r.dlogits).all(1).tolist() == [True, True, True, False] * 2 and bool(torch.isnan(r.loss))
