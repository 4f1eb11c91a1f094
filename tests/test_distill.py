"""distill_loss_fwd_bwd and DistillLoss against the 64-bit oracle."""
import numpy as np
import pytest
import torch

import oracle
import paper_2605_12070_amd as P
from operator_helpers import DEV, GRAD, KL, U, near, rows, values_of

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def record(z, k, seed, tau=1.0, short=True, kept=0.8):
    """k distinct tokens per row, likely ones among them, other values; every third record shorter."""
    T, V = z.shape
    rng = np.random.default_rng(seed)
    zz = np.nan_to_num(values_of(z), neginf=-50.0, posinf=50.0)
    ids = np.empty((T, k), dtype=np.int32)
    for t in range(T):
        best = np.argsort(-zz[t])[:max(1, k // 2)]
        rest = rng.choice(V, size=min(V, 2 * k), replace=False)
        ids[t] = np.concatenate([best, rest[~np.isin(rest, best)]])[:k]
        rng.shuffle(ids[t])
    values = (np.take_along_axis(zz, ids.astype(np.int64), 1) + rng.normal(0, 0.7, (T, k))).astype(np.float32)
    if short and k > 2:
        ids[::3, k - k // 3:] = -1
    x = np.where(ids >= 0, values.astype(np.float64) / tau, -np.inf)
    lse = (oracle.dppo_oracle.row_logsumexp(x) - np.log(kept)).astype(np.float32)
    return torch.from_numpy(values).to(DEV), torch.from_numpy(ids).to(DEV), torch.from_numpy(lse).to(DEV)


def compare(r, z, values, ids, lse, mask=None, ts=None, zvals=None, **kw):
    ref = oracle.distill_loss(values_of(z) if zvals is None else zvals, values.cpu().numpy(), ids.cpu().numpy(),
                              None if lse is None else lse.cpu().double().numpy(),
                              None if mask is None else mask.cpu().numpy(),
                              None if ts is None else ts.cpu().double().numpy(), **kw)
    near(r.kl.cpu().numpy(), ref["kl"], KL * np.maximum(1, np.abs(np.nan_to_num(ref["kl"]))), "kl")
    assert np.array_equal(r.flags.cpu().numpy(), ref["flags"])
    assert r.stats.cpu().tolist() == [ref["n_valid"], 0, 0, 0, ref["n_bad"]]
    if np.isfinite(ref["loss"]):
        size = np.abs(ref["kl"]).max(initial=0.0)
        scale = abs(kw.get("loss_scale", 1.0)) * (1 if kw.get("scale_mode") != "const" else len(ref["kl"]))
        big = 1.0 if ts is None else float(ts.max())
        near(r.loss.cpu().numpy(), [ref["loss"]], 2 * KL * max(1.0, size) * scale * big, "loss")
    if r.dlogits is not None:
        tol = U[r.dlogits.dtype] * np.abs(ref["dlogits"]) + GRAD * ref["slack"] + 2.0 ** -126
        near(values_of(r.dlogits), ref["dlogits"], tol, "dlogits")
    return ref


def run(z, k, tail, seed, tau=1.0, mask=None, ts=None, dlogits=None, **kw):
    values, ids, lse = record(z, k, seed, tau)
    lse = lse if tail else None
    r = P.distill_loss_fwd_bwd(z, values, ids, lse, mask, ts, temperature=tau, dlogits=dlogits, **kw)
    torch.cuda.synchronize()
    compare(r, z, values, ids, lse, mask, ts, tau=tau, **kw)
    return r


# every workgroup shape and the lengths around its capacity
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,V,k", [
    (1, 1, 1), (2, 3, 2), (3, 8, 8), (4, 31, 5), (5, 1000, 16), (3, 2049, 256), (3, 4096, 7), (3, 8200, 64),
    (2, 16385, 100), (3, 32768, 33), (2, 50257, 128), (2, 65537, 20), (2, 98304, 64), (2, 151936, 64),
    (2, 155649, 256), (2, 200003, 31), (1, 262144, 64), (1, 300000, 12),
])
def test_random_rows(dtype, T, V, k, tail):
    print(f"[case] distill {dtype} T={T} V={V} k={k} tail={tail}", flush=True)
    run(rows(T, V, dtype, seed=T + V + k), k, tail, seed=V, tau=1.0 if V % 2 else 1.7)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("V", [1201, 33000])
@pytest.mark.parametrize("offset,d_offset", [(0, 0), (1, 1), (3, 0), (0, 5), (2, 3)])
def test_strides_offsets_and_guards(dtype, V, offset, d_offset):
    """Rows at any offset, dlogits at another one; nothing outside the rows is written."""
    print(f"[case] distill {dtype} V={V} offset={offset} d_offset={d_offset}", flush=True)
    z = rows(5, V, dtype, seed=3, ld=V + 5, offset=offset)
    buf = torch.full((5 * (V + 9) + 64,), 55.0, dtype=dtype, device=DEV)
    d = buf.as_strided((5, V), (V + 9, 1), d_offset)
    mask = torch.tensor([1, 0, 1, 1, 0], dtype=torch.uint8, device=DEV)
    ts = torch.tensor([0.6, 1.1, 0.9, 1.4, 0.7], device=DEV)
    r = run(z, 40, True, seed=8, mask=mask, ts=ts, dlogits=d)
    assert r.dlogits is d
    out = torch.ones_like(buf, dtype=torch.bool)
    out.as_strided((5, V), (V + 9, 1), d_offset).fill_(False)
    assert bool((buf[out] == 55.0).all())


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("V", [513, 40000, 170001])
def test_in_place_and_scales(dtype, V):
    print(f"[case] distill in place {dtype} V={V}", flush=True)
    z = rows(4, V, dtype, seed=2)
    zvals = values_of(z)
    values, ids, lse = record(z, 50, 4, 0.8)
    ts = torch.tensor([0.5, 1.0, 0.0, 3.0], device=DEV)
    kw = dict(scale_mode="const", loss_scale=-0.25)
    r = P.distill_loss_fwd_bwd(z, values, ids, lse, None, ts, temperature=0.8, dlogits=z, **kw)
    torch.cuda.synchronize()
    compare(r, z, values, ids, lse, None, ts, zvals=zvals, tau=0.8, **kw)


def test_forward_only_gives_the_same_loss():
    z = rows(9, 30001, BF, seed=1)
    values, ids, lse = record(z, 64, 1)
    a = P.distill_loss_fwd_bwd(z, values, ids, lse)
    b = P.distill_loss_fwd_bwd(z, values, ids, lse, want_dlogits=False)
    assert b.dlogits is None
    assert torch.equal(a.kl, b.kl) and torch.equal(a.loss, b.loss) and torch.equal(a.stats, b.stats)


@pytest.mark.parametrize("T", [3, 70, 2000, 70000])
@pytest.mark.parametrize("masked", ["none", "some", "all"])
def test_batches_and_masks(T, masked):
    print(f"[case] distill T={T} masked={masked}", flush=True)
    V, k = 40, 6
    z = rows(T, V, F32, seed=T)
    g = torch.Generator().manual_seed(T)
    ids = torch.rand(T, V, generator=g).argsort(1)[:, :k].to(torch.int32).contiguous().to(DEV)
    values = torch.randn(T, k, generator=g).to(DEV)
    mask = {"none": None, "all": torch.zeros(T, dtype=torch.uint8, device=DEV),
            "some": (torch.rand(T, generator=g) < 0.6).to(torch.uint8).to(DEV)}[masked]
    r = P.distill_loss_fwd_bwd(z, values, ids, None, mask)
    torch.cuda.synchronize()
    m = np.ones(T) if mask is None else mask.cpu().numpy() != 0
    n = max(1, int(m.sum()))
    zz, tv, ii = values_of(z), values.cpu().double().numpy(), ids.cpu().numpy().astype(np.int64)
    logq = zz - np.log(np.exp(zz).sum(1, keepdims=True))
    p = np.exp(tv) / np.exp(tv).sum(1, keepdims=True)
    kl = (p * (np.log(p) - np.take_along_axis(logq, ii, 1))).sum(1) * m
    d = np.exp(logq)
    np.put_along_axis(d, ii, np.take_along_axis(d, ii, 1) - p, 1)
    near(r.kl.cpu().numpy(), kl, KL * np.maximum(1, np.abs(kl)), "kl")
    near(values_of(r.dlogits), d * m[:, None] / n, 2 * GRAD / n, "dlogits")
    near(r.loss.cpu().numpy(), [kl.sum() / n], KL * max(1, np.abs(kl).max()), "loss")
    assert r.stats.cpu().tolist() == [int(m.sum()), 0, 0, 0, 0]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("V", [90, 20000, 160001])
def test_unusual_records(dtype, tail, V):
    """Empty records, a token listed twice and three times, values of -inf, ids out of range, a
    record that holds the whole vocabulary's mass, the row's ends, one chunk full of the record."""
    print(f"[case] distill records {dtype} tail={tail} V={V}", flush=True)
    k = 24
    z = rows(9, V, dtype, seed=V)
    values, ids, lse = record(z, k, 5, short=False)
    ids[0] = -1
    ids[1, 3] = ids[1, 9]
    ids[1, 11] = ids[1, 9]
    values[2, 4:] = -float("inf")
    ids[3, 7] = V
    ids[4, 0] = -2
    lse[5] -= 5.0                               # probabilities that add up to more than 1
    ids[6] = torch.arange(k, device=DEV)
    ids[7] = torch.arange(V - k, V, device=DEV)
    ids[8] = 40 + torch.arange(k, device=DEV) // 2
    values[8, 5] = -float("inf")
    r = P.distill_loss_fwd_bwd(z, values, ids, lse if tail else None)
    torch.cuda.synchronize()
    compare(r, z, values, ids, lse if tail else None)
    assert bool((r.dlogits[3] == 0).all()) and r.flags.cpu()[3] == 9
    if not tail:
        assert bool((r.dlogits[0] == 0).all())


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("V", [70, 9001])
def test_student_extremes(dtype, tail, V):
    """A student all but sure of one token, in the record and outside it; masked logits (-inf and the
    type's lowest value); a record's token at -inf; rows of -inf, NaN, +inf."""
    print(f"[case] distill student {dtype} tail={tail} V={V}", flush=True)
    z = rows(9, V, dtype, seed=V)
    values, ids, lse = record(z, 8, 5, short=False)
    z[0, int(ids[0, 2])] = 40.0
    free = [v for v in range(V) if v not in set(ids[1].tolist())][3]
    z[1, free] = 40.0
    z[2, 20:] = -float("inf")
    z[3, 20:] = torch.finfo(dtype).min
    z[4, int(ids[4, 1])] = -float("inf")
    z[5] = -float("inf")
    z[6, 5] = float("nan")
    z[7, 6] = float("inf")
    ids[2] = torch.arange(2, 10, device=DEV)
    ids[3] = torch.arange(2, 10, device=DEV)
    r = P.distill_loss_fwd_bwd(z, values, ids, lse if tail else None)
    torch.cuda.synchronize()
    got = (r.kl.cpu().numpy(), values_of(r.dlogits))
    for t in (5, 6, 7):                        # data errors stay visible
        assert not np.isfinite(got[0][t])
        assert np.isnan(got[1][t]).all()
    assert got[0][4] == np.inf
    keep = torch.tensor([0, 1, 2, 3, 8], device=DEV)
    sub = P.distill_loss_fwd_bwd(z[keep], values[keep], ids[keep], lse[keep] if tail else None)
    torch.cuda.synchronize()
    compare(sub, z[keep], values[keep], ids[keep], lse[keep] if tail else None)


def test_autograd_scales_and_matches_differences():
    z = rows(6, 37, F32, seed=5).contiguous()
    values, ids, lse = record(z, 5, 6)
    mask = torch.tensor([1, 1, 0, 1, 1, 1], dtype=torch.uint8, device=DEV)
    leaf = z.clone().requires_grad_(True)
    loss, kl, stats = P.DistillLoss.apply(leaf, values, ids, lse, mask, None, dict(temperature=1.3))
    (3.0 * loss).backward()
    r = P.distill_loss_fwd_bwd(z, values, ids, lse, mask, temperature=1.3)
    assert torch.equal(leaf.grad, 3.0 * r.dlogits) and torch.equal(kl, r.kl) and torch.equal(loss, r.loss[0])
    assert not kl.requires_grad and not stats.requires_grad
    # differences of the oracle's loss on the kernel's inputs
    args = (values.cpu().numpy(), ids.cpu().numpy(), lse.cpu().double().numpy(), mask.cpu().numpy(), None, 1.3)
    zz, h = values_of(z), 1e-5
    for t, v in ((0, 3), (1, int(ids[1, 0])), (2, 5), (5, int(ids[5, 4]))):
        e = np.zeros_like(zz)
        e[t, v] = h
        slope = (oracle.distill_loss(zz + e, *args)["loss"] - oracle.distill_loss(zz - e, *args)["loss"]) / (2 * h)
        assert abs(slope - float(r.dlogits[t, v])) < 1e-6


def test_autograd_without_gradient_for_the_loss_and_empty_batch():
    z = rows(4, 50, BF, seed=5).contiguous().requires_grad_(True)
    values, ids, lse = record(z, 5, 6)
    loss, kl, stats = P.DistillLoss.apply(z, values, ids, None, None, None, None)
    (g,) = torch.autograd.grad(loss * 0.0, z)
    assert bool((g == 0).all())
    e = P.distill_loss_fwd_bwd(z.detach()[:0], values[:0], ids[:0], lse[:0])
    assert float(e.loss) == 0.0 and e.stats.cpu().tolist() == [0] * 5 and e.dlogits.shape == (0, 50)


def test_another_stream_and_the_same_bits_again():
    z = rows(700, 33333, BF, seed=4)
    values, ids, lse = record(z[:7], 30, 1)
    values, ids, lse = (t.repeat(100, *[1] * (t.dim() - 1)).contiguous() for t in (values, ids, lse))
    a = P.distill_loss_fwd_bwd(z, values, ids, lse)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        b = P.distill_loss_fwd_bwd(z, values, ids, lse)
    s.synchronize()
    for x, y in ((a.loss, b.loss), (a.kl, b.kl), (a.dlogits, b.dlogits), (a.stats, b.stats)):
        assert torch.equal(x, y)


# rows enough for the shapes of fewer threads: their capacities, rows that start anywhere, more rows than
# fit on the device at once
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("chunks,T,k", [
    (3, 600, 2), (250, 600, 20), (40, 20000, 5), (256, 9000, 64), (511, 700, 100), (900, 5000, 9), (1024, 600, 256),
    (2047, 530, 30), (4095, 1600, 65), (4096, 520, 3), (6143, 530, 200), (8191, 530, 12),
])
def test_many_rows(dtype, chunks, T, k):
    V = chunks * (8 if dtype == BF else 4) - 1 + chunks % 3
    print(f"[case] distill rows {dtype} T={T} V={V} k={k}", flush=True)
    few = 7
    z7 = rows(few, V, dtype, seed=V)
    values, ids, lse = record(z7, k, V)
    z = z7[torch.arange(T, device=DEV) % few]                  # rows of an odd length start anywhere
    many = [t[torch.arange(T, device=DEV) % few] for t in (values, ids, lse)]
    mask = (torch.arange(T, device=DEV) % 11 != 3).to(torch.uint8)
    ref = oracle.distill_loss(values_of(z7), values.cpu().numpy(), ids.cpu().numpy(), lse.cpu().double().numpy(),
                              scale_mode="const")
    d = torch.full((T, V + 3), 5.0, dtype=dtype, device=DEV)
    r = P.distill_loss_fwd_bwd(z, *many, mask, scale_mode="const", dlogits=d[:, 1:V + 1])
    on = mask.bool()
    kl = torch.from_numpy(ref["kl"]).to(DEV)
    want = torch.from_numpy(ref["dlogits"]).to(DEV)
    tol = U[dtype] * want.abs() + GRAD * torch.from_numpy(ref["slack"]).to(DEV) + 2.0 ** -126
    assert bool((r.flags == mask).all()) and int(r.stats[0]) == int(on.sum())
    assert bool((d[:, 0] == 5.0).all()) and bool((d[:, V + 1:] == 5.0).all())
    for c in range(few):                                       # the rows of one content
        t = torch.arange(c, T, few, device=DEV)
        live, dead = t[on[t]], t[~on[t]]
        assert float((r.kl[live].double() - kl[c]).abs().max()) <= KL * max(1.0, abs(float(kl[c])))
        assert bool((r.kl[dead] == 0).all()) and bool((d[dead, 1:V + 1] == 0).all())
        for part in live.split(64):
            assert bool(((d[part, 1:V + 1].double() - want[c]).abs() <= tol[c]).all()), (c, part)
    total = sum(float(kl[c]) * int(on[torch.arange(c, T, few, device=DEV)].sum()) for c in range(few))
    assert abs(float(r.loss) - total) <= 2 * KL * T * max(1.0, float(kl.abs().max()))
    in_place = P.distill_loss_fwd_bwd(z, *many, mask, scale_mode="const", dlogits=z)
    got = in_place.dlogits[on][:50].double()
    c = (torch.arange(T, device=DEV) % few)[on][:50]
    assert bool(((got - want[c]).abs() <= tol[c]).all())
