"""Performance cases of the vocabulary-row operators around the loss stage: the record of a
teacher's top logits, the distillation loss that reads it, and the verification of drafted tokens.

Kinds of case (the "kind" entry) and what they stand for:
  top      the k largest logits of every row with the row's log-sum-exp: what a teacher's scoring
           pass keeps of its logits, or a serving step's top candidates
  distill  one training step's distillation loss against such records, with its gradient: the
           plain call ("call") or inside a model's autograd graph ("autograd")
  verify   one step of a rollout by speculative decoding: drafted tokens accepted or replaced
           against the policy's logits, and the log-probs of what was emitted

`own` chooses between the package's entry points and the same operators in elementary torch
operations.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
ACCUM = 0.25                     # gradient-accumulation factor of the autograd cases
TAIL_FLOOR = 2.0 ** -24          # least tail mass a student is given
LARGEST = 8192 * 151936 * 2      # bytes of the largest logits matrix
VERIFY_LARGEST = 256 * 9 * 151936 * 2


# ------------------------------------------------------------------ the cases
def listed():
    return [
        # a decoding step's candidates, eight sequences: latency counts
        dict(name="top_decode", kind="top", dtype="bf16", T=8, V=32000, k=20, tau=1.0),
        # one sequence's token over the longest rows
        dict(name="top_one_long_row", kind="top", dtype="f32", T=1, V=262144, k=64, tau=0.7),
        # a teacher that returns fp32 logits of an odd vocabulary, rows at any offset
        dict(name="top_f32_odd_vocab", kind="top", dtype="f32", T=2048, V=50257, k=128, tau=1.0),
        # a teacher's scoring pass at full size
        dict(name="top_large_vocab", kind="top", dtype="bf16", T=8192, V=151936, k=64, tau=1.0),
        # the smallest training step
        dict(name="distill_tiny_f32", kind="distill", api="call", dtype="f32", T=256, V=1024, k=16,
             tau=1.0, tail=False, mask=0.0),
        # a drafter's training step inside its autograd graph, tool output masked, softened logits
        dict(name="distill_autograd", kind="distill", api="autograd", dtype="bf16", T=4096, V=32000,
             k=32, tau=2.0, tail=False, mask=0.4),
        # a trainer that upcasts its logits: fp32 rows of an odd vocabulary, wide records with a tail
        dict(name="distill_f32_odd_vocab", kind="distill", api="call", dtype="f32", T=4096, V=50257,
             k=128, tau=1.0, tail=True, mask=0.0),
        # the full vocabulary, a tail bucket
        dict(name="distill_large_vocab", kind="distill", api="call", dtype="bf16", T=8192, V=151936,
             k=64, tau=1.0, tail=True, mask=0.0),
        # a single interactive sequence
        dict(name="verify_one", kind="verify", dtype="bf16", B=1, D=4, V=32000, drafts="logits",
             ragged=False, tau=1.0),
        # greedy or n-gram drafts without a distribution, ragged, fp32 rows of an odd vocabulary
        dict(name="verify_tokens_f32", kind="verify", dtype="f32", B=64, D=8, V=50257,
             drafts="tokens", ragged=True, tau=0.8),
        # a small rollout batch
        dict(name="verify_rollout", kind="verify", dtype="bf16", B=32, D=5, V=151936, drafts="logits",
             ragged=True, tau=1.0),
        # a full rollout batch
        dict(name="verify_large", kind="verify", dtype="bf16", B=256, D=4, V=151936, drafts="logits",
             ragged=False, tau=1.0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["top", "top", "distill", "distill", "verify", "verify"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    es = 4 if dtype == "f32" else 2
    V = _log_int(rng, 1000, 262144)
    if rng.random() < 0.5:
        V = 16 * (V // 16)
    tau = rng.choice([1.0, 1.0, 0.7, 2.0])
    if kind == "verify":
        D = rng.randint(1, 8)
        drafts = rng.choice(["logits", "logits", "tokens"])
        B = _log_int(rng, 1, 512)
        B = max(1, min(B, VERIFY_LARGEST // ((2 * D + 1) * V * es)))
        return dict(kind=kind, dtype=dtype, B=B, D=D, V=V, drafts=drafts,
                    ragged=rng.random() < 0.5, tau=tau)
    k = min(_log_int(rng, 1, 256), V // 4)
    if kind == "top":
        T = max(1, min(_log_int(rng, 1, 8192), LARGEST // (V * es)))
        return dict(kind=kind, dtype=dtype, T=T, V=V, k=k, tau=tau)
    T = max(1, min(_log_int(rng, 64, 8192), LARGEST // (V * es)))
    return dict(kind=kind, api=rng.choice(["call", "call", "autograd"]), dtype=dtype, T=T, V=V, k=k,
                tau=tau, tail=rng.random() < 0.5, mask=rng.choice([0.0, 0.4]))


# ------------------------------------------------------------------ inputs
def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _slices(rows, V):
    """Rows in slices of at most 1 GiB of float32."""
    n = max(1, min(rows, (1 << 28) // V))
    return [slice(a, min(rows, a + n)) for a in range(0, rows, n)]


def _logits(rows, V, dtype, gen):
    """N(0, 3^2) logits; half of the rows have one entry up to 16 above its place (a confident
    token)."""
    z = torch.empty(rows, V, dtype=dtype, device=DEV)
    for s in _slices(rows, V):
        z[s] = (3.0 * torch.randn(s.stop - s.start, V, generator=gen, device=DEV)).to(dtype)
    at = torch.randint(0, V, (rows, 1), generator=gen, device=DEV)
    up = 16.0 * torch.rand(rows, 1, generator=gen, device=DEV)
    up *= torch.rand(rows, 1, generator=gen, device=DEV) < 0.5
    return z.scatter_add_(1, at, up.to(dtype))


def _teacher(z, case, gen):
    """A teacher's record beside the student's rows z: k distinct tokens the student finds likely
    (the best of each of k stretches of the vocabulary), other values, a share of the mass left
    out; one row in sixteen has a shorter record, its last entries empty (id -1)."""
    (T, V), k, tau = z.shape, case["k"], case["tau"]
    w = V // k
    ids = torch.empty(T, k, dtype=torch.int64, device=DEV)
    for s in _slices(T, V):
        ids[s] = z[s, :w * k].view(-1, k, w).argmax(2)
    ids += w * torch.arange(k, device=DEV)
    values = z.gather(1, ids).float() + 0.5 * torch.randn(T, k, generator=gen, device=DEV)
    values, order = values.sort(dim=1, descending=True)
    ids = ids.gather(1, order)
    if k >= 8:
        short = torch.rand(T, 1, generator=gen, device=DEV) < 1 / 16
        ids = ids.masked_fill(short & (torch.arange(k, device=DEV) >= k - k // 4), -1)
    left = 0.02 + 0.38 * torch.rand(T, generator=gen, device=DEV)
    kept = torch.where(ids >= 0, values / tau, torch.full_like(values, -math.inf))
    lse = torch.logsumexp(kept, 1) - torch.log1p(-left)
    return values.contiguous(), ids.to(torch.int32), lse


def _mask(T, share, gen):
    """Spans of tool output (0) among a batch's tokens."""
    if share == 0.0:
        return torch.ones(T, dtype=torch.uint8, device=DEV)
    span = torch.arange(T, device=DEV) % int(300 / (1 - share))
    shift = int(torch.randint(0, 300, (1,), generator=gen, device=DEV))
    return (span.roll(shift) < 300).to(torch.uint8) if T > 600 else \
        (torch.rand(T, generator=gen, device=DEV) >= share).to(torch.uint8)


def _drafts(z, case, gen):
    """Drafted tokens beside the policy's rows z [B, D + 1, V]: sampled from a draft model whose
    logits are the policy's with N(0, 0.7^2) noise, or the noisy logits' best token."""
    B, D, V, tau = case["B"], case["D"], case["V"], case["tau"]
    q = torch.empty(B * D, V, dtype=z.dtype, device=DEV)
    ids = torch.empty(B * D, dtype=torch.int64, device=DEV)
    rows = z[:, :D].reshape(B * D, V)
    for s in _slices(B * D, V):
        x = rows[s].float()
        x = (x + 0.7 * torch.randn(x.shape, generator=gen, device=DEV)).to(z.dtype)
        q[s] = x
        x = x.float() / tau
        if case["drafts"] == "logits":
            x -= torch.empty_like(x).exponential_(generator=gen).log_()
        ids[s] = x.argmax(1)
    return q.view(B, D, V), ids.view(B, D)


def prepare(case, seed):
    gen = _gen(seed)
    s = dict(case=case)
    if case["kind"] == "verify":
        B, D, V = case["B"], case["D"], case["V"]
        s["z"] = _logits(B * (D + 1), V, _dtype(case), gen).view(B, D + 1, V)
        q, s["ids"] = _drafts(s["z"], case, gen)
        s["q"] = q if case["drafts"] == "logits" else None
        s["u"] = torch.rand(B, D, generator=gen, device=DEV)
        s["u_new"] = torch.rand(B, generator=gen, device=DEV)
        s["n"] = torch.randint(0, D + 1, (B,), generator=gen, device=DEV, dtype=torch.int32) \
            if case["ragged"] else None
        return s
    s["z"] = _logits(case["T"], case["V"], _dtype(case), gen)
    if case["kind"] == "distill":
        s["values"], s["ids"], s["lse"] = _teacher(s["z"], case, gen)
        if not case["tail"]:
            s["lse"] = None
        s["mask"] = _mask(case["T"], case["mask"], gen)
        if case["api"] == "autograd":
            s["z"].requires_grad_(True)
    return s


# ------------------------------------------------------------------ one pass
def _plain_top(z, k, tau):
    x = z.float()
    bits = (x + 0.0).view(torch.int32)                    # -0 becomes +0
    key = bits ^ ((bits >> 31) & 0x7FFFFFFF)              # ordered like the values
    # keys that differ: equal values go by their index, the lowest first
    key = (key.long() << 32) + torch.arange(z.shape[1] - 1, -1, -1, device=z.device)
    ids = z.shape[1] - 1 - (torch.topk(key, k, dim=1).values & 0xFFFFFFFF)
    x = x / tau
    m = x.amax(1, keepdim=True)
    lse = m[:, 0] + torch.log(torch.exp(x - m).sum(1))
    return dict(values=z.gather(1, ids).float(), ids=ids.to(torch.int32), lse=lse)


def _plain_distill(z, values, ids, lse, mask, tau):
    T, V = z.shape
    x = z.float() / tau
    m = x.amax(1, keepdim=True)
    logq = x - (m + torch.log(torch.exp(x - m).sum(1, keepdim=True)))
    q = torch.exp(logq)
    held = ids >= 0
    at = ids.clamp_min(0).long()
    t = torch.where(held, values / tau, torch.full_like(values, -math.inf))
    if lse is None:
        top = t.amax(1, keepdim=True)
        c = top + torch.log(torch.exp(t - top).sum(1, keepdim=True))
    else:
        c = lse[:, None]
    p = torch.exp(t - c)
    logq_at = logq.gather(1, at)
    zero = torch.zeros_like(p)
    kl = torch.where(p > 0, p * (t - c - logq_at), zero).sum(1)
    P = p.sum(1)
    q_at = torch.where(held, q.gather(1, at), zero)
    rest = q.scatter_add(1, at, -q_at)                    # the softmax with 0 at the record's tokens
    inside, outside = P, P
    if lse is not None:
        Q = q_at.sum(1)
        # the mass outside the record as a sum of its own: 1 - Q would lose it next to 1
        Pt, Qt = (1 - P).clamp_min(0), rest.sum(1).clamp_min(TAIL_FLOOR)
        kl = kl + torch.where(Pt > 0, Pt * torch.log(Pt / Qt), torch.zeros_like(Pt))
        inside, outside = P + Pt, P - Pt * Q / Qt
    on = mask != 0
    n = on.sum()
    s = torch.where(on, 1.0 / n.clamp_min(1), torch.zeros_like(kl))
    d = rest * (s / tau * outside)[:, None]
    d.scatter_add_(1, at, torch.where(held, (s / tau)[:, None] * (inside[:, None] * q_at - p), zero))
    kl = torch.where(on, kl, torch.zeros_like(kl))
    stats = torch.zeros(5, dtype=torch.int32, device=z.device)
    stats[0] = n
    return dict(loss=(s.double() * kl.double()).sum()[None].float(), kl=kl, stats=stats, dlogits=d.to(z.dtype))


def _plain_verify(z, ids, u, u_new, q, n, tau):
    B, D1, V = z.shape
    D = D1 - 1
    # decisions next to a border: 64 bits
    x = z.double() / tau
    x = x - x.amax(2, keepdim=True)
    logp = x - torch.log(torch.exp(x).sum(2, keepdim=True))
    p_at = torch.exp(logp[:, :D].gather(2, ids[..., None])[..., 0])
    if q is None:
        qd = torch.zeros(B, D, V, dtype=torch.float64, device=z.device).scatter_(2, ids[..., None], 1.0)
    else:
        y = q.double() / tau
        y = y - y.amax(2, keepdim=True)
        y = torch.exp(y)
        qd = y / y.sum(2, keepdim=True)
    q_at = qd.gather(2, ids[..., None])[..., 0]
    pos = torch.arange(D1, device=z.device)
    n = torch.full((B,), D, device=z.device) if n is None else n.long()
    ok = (u.double() * q_at < p_at) & (pos[:D] < n[:, None])
    acc = ok.long().cumprod(1).sum(1)
    at = acc[:, None, None].expand(B, 1, V)
    p_n = torch.exp(logp.gather(1, at)[:, 0])
    q_n = qd.gather(1, at.clamp_max(D - 1))[:, 0] * (acc < n)[:, None]
    r = (p_n - q_n).clamp_min(0)
    r = torch.where(r.sum(1, keepdim=True) > 0, r, p_n)
    c = r.cumsum(1)
    new = (c <= u_new.double()[:, None] * c[:, -1:]).sum(1)
    new = torch.minimum(new, torch.where(r > 0, torch.arange(V, device=z.device), -1).amax(1))
    full = torch.cat([ids, ids[:, :1]], 1)
    here = pos[None] == acc[:, None]
    tokens = torch.where(here, new[:, None], full).masked_fill(pos[None] > acc[:, None], -1)
    lp = logp.gather(2, tokens.clamp_min(0)[..., None])[..., 0].masked_fill(tokens < 0, 0.0)
    return dict(accepted=acc.to(torch.int32), tokens=tokens, logp=lp.float())


def run(s):
    case, z = s["case"], s["z"]
    kind, tau = case["kind"], case["tau"]
    if own:
        import paper_2605_12070_amd as P
        if kind == "top":
            r = P.top_logits(z, case["k"], temperature=tau)
            return dict(values=r.values, ids=r.ids, lse=r.lse)
        if kind == "verify":
            r = P.verify_drafts(z, s["ids"], s["u"], s["u_new"], s["q"], s["n"], temperature=tau)
            return dict(accepted=r.accepted, tokens=r.tokens, logp=r.logp)
        if case["api"] == "call":
            r = P.distill_loss_fwd_bwd(z, s["values"], s["ids"], s["lse"], s["mask"], temperature=tau)
            return dict(loss=r.loss, kl=r.kl, stats=r.stats, dlogits=r.dlogits)
        loss, kl, stats = P.DistillLoss.apply(z, s["values"], s["ids"], s["lse"], s["mask"], None,
                                              dict(temperature=tau))
        (g,) = torch.autograd.grad(loss * ACCUM, z)
        return dict(loss=loss.detach(), kl=kl, stats=stats, dlogits=g)
    z = z.detach()
    if kind == "top":
        return _plain_top(z, case["k"], tau)
    if kind == "verify":
        return _plain_verify(z, s["ids"], s["u"], s["u_new"], s["q"], s["n"], tau)
    r = _plain_distill(z, s["values"], s["ids"], s["lse"], s["mask"], tau)
    if case["api"] == "autograd":
        r.update(loss=r["loss"][0], dlogits=r["dlogits"] * ACCUM)
    return r


# ------------------------------------------------------------------ what a pass needs
def work(case):
    es = 4 if case["dtype"] == "f32" else 2
    V = case["V"]
    if case["kind"] == "top":
        T, k = case["T"], case["k"]
        return dict(bytes=T * (V * es + 8 * k + 4), flops=4 * T * V)
    if case["kind"] == "distill":
        T, k = case["T"], case["k"]
        keep = 1.0 - case["mask"]
        again = 2 * T * V * es * (case["api"] == "autograd")   # the upstream factor comes later
        return dict(bytes=int(T * V * es * (1.0 + keep) + again + T * (8 * k + 10)), flops=6 * T * V)
    # the rows up to the first rejection; about three drafts in four are accepted here
    D = case["D"] if not case["ragged"] else case["D"] / 2
    rows = (1 - 0.75 ** (D + 1)) / 0.25
    rows = rows * (2 if case["drafts"] == "logits" else 1)
    return dict(bytes=int(case["B"] * (rows * V * es + 28 * (case["D"] + 1))),
                flops=int(case["B"] * rows * V * 4))


# ------------------------------------------------------------------ 64-bit values
def _exact_distill(s):
    case, z = s["case"], s["z"].detach()
    (T, V), tau = z.shape, case["tau"]
    kl = torch.zeros(T, dtype=torch.float64, device=DEV)
    d = torch.zeros(T, V, dtype=torch.float64, device=DEV)
    on = s["mask"] != 0
    scale = 1.0 / max(1, int(on.sum()))
    for c in on.nonzero()[:, 0].split(max(1, (1 << 27) // V)):
        logq = torch.log_softmax(z[c].double() / tau, 1)
        ids = s["ids"][c].long()
        t = (s["values"][c].double() / tau).masked_fill(ids < 0, -math.inf)
        logp = torch.log_softmax(t, 1) if s["lse"] is None else t - s["lse"][c].double()[:, None]
        p = logp.exp()
        dense = torch.zeros_like(logq).scatter_add_(1, ids.clamp_min(0), p)      # the record as a row
        member = torch.zeros_like(logq).scatter_add_(1, ids.clamp_min(0), (ids >= 0).double())
        q = logq.exp()
        cross = (p * logq.gather(1, ids.clamp_min(0))).sum(1)
        kl[c] = torch.special.entr(p).sum(1).neg() - cross
        if s["lse"] is None:
            d[c] = q - dense
        else:
            rest = 1.0 - p.sum(1)
            left = torch.where(member > 0, torch.zeros_like(q), q).sum(1).clamp_min(TAIL_FLOOR)
            kl[c] += torch.where(rest > 0, rest * (rest / left).log(), torch.zeros_like(rest))
            d[c] = torch.where(member > 0, q - dense, q * (1.0 - rest / left)[:, None])
        d[c] *= scale / tau
    loss = kl.sum() * scale
    if case["api"] == "autograd":
        return dict(loss=loss, kl=kl, stats=None, dlogits=d.mul_(ACCUM))
    return dict(loss=loss[None], kl=kl, stats=None, dlogits=d)


def _exact_verify(s):
    """One sequence after another, one draft after another."""
    case, tau = s["case"], s["case"]["tau"]
    B, D = case["B"], case["D"]
    out = torch.zeros(B, D + 1, dtype=torch.float64)
    u, u_new, ids = s["u"].double().cpu(), s["u_new"].double().cpu(), s["ids"].cpu()
    n = [D] * B if s["n"] is None else s["n"].tolist()
    for b in range(B):
        for i in range(D + 1):
            lp = torch.log_softmax(s["z"][b, i].double() / tau, 0)
            r = lp.exp()
            if i < n[b]:
                x = int(ids[b, i])
                if s["q"] is None:
                    q = torch.zeros_like(r)
                    q[x] = 1.0
                else:
                    q = torch.softmax(s["q"][b, i].double() / tau, 0)
                lp_x, p_x, q_x = torch.stack([lp[x], r[x], q[x]]).tolist()
                if float(u[b, i]) * q_x < p_x:
                    out[b, i] = lp_x
                    continue
                r = (r - q).relu()
            c = torch.cumsum(r, 0)
            v = int(torch.searchsorted(c, (c[-1] * float(u_new[b]))[None], right=True))
            out[b, i] = float(lp[v])
            break
    return dict(accepted=None, tokens=None, logp=out.to(DEV))


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "distill":
        return _exact_distill(s)
    if case["kind"] == "verify":
        return _exact_verify(s)
    z = s["z"]
    values = torch.empty(case["T"], case["k"], dtype=torch.float64, device=DEV)
    lse = torch.empty(case["T"], dtype=torch.float64, device=DEV)
    for c in _slices(case["T"], case["V"]):
        values[c] = torch.topk(z[c].double(), case["k"], dim=1).values
        lse[c] = torch.logsumexp(z[c].double() / case["tau"], 1)
    return dict(values=values, ids=None, lse=lse)
