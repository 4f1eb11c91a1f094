"""What top_logits, distill_loss_fwd_bwd and verify_drafts refuse, at the C boundary (no GPU: every
case fails its host-side check) and in the binding."""
import ctypes as C
import os

import pytest
import torch

import paper_2605_12070_amd as P
from paper_2605_12070_amd import _lib

pytestmark = pytest.mark.skipif(not os.path.exists(_lib.LIB_PATH), reason="libdppo.so not built")

FAKE = 0x10000  # never dereferenced
INVALID = 1
NAN, INF = float("nan"), float("inf")


def refused(status, words):
    assert status == INVALID
    text = _lib.lib().dppo_last_error().decode()
    assert words in text, text


# ---------------------------------------------------------------- top_logits
def top(**kw):
    a = dict(logits=FAKE, dtype=_lib.DPPO_BF16, T=4, V=1000, ld=1000, k=8, temperature=1.0, values=FAKE, ids=FAKE,
             lse=FAKE, workspace=None, workspace_bytes=0, stream=None)
    a.update(kw)
    return _lib.lib().top_logits(*a.values())


@pytest.mark.parametrize("kw,words", [
    (dict(logits=None), "logits"),
    (dict(logits=FAKE + 1), "aligned"),
    (dict(dtype=_lib.DPPO_F32, logits=FAKE + 2), "aligned"),
    (dict(dtype=7), "dtype"),
    (dict(T=-1), "T"),
    (dict(T=1 << 31), "T"),
    (dict(V=0), "V"),
    (dict(V=(1 << 28) + 1, ld=1 << 29), "V"),
    (dict(ld=999), "stride"),
    (dict(k=0), "k = 0"),
    (dict(k=-3), "k = -3"),
    (dict(k=257), "k = 257"),
    (dict(V=5, ld=5, k=6), "k = 6"),
    (dict(temperature=0.0), "temperature"),
    (dict(temperature=-1.0), "temperature"),
    (dict(temperature=NAN), "temperature"),
    (dict(temperature=INF), "temperature"),
    (dict(temperature=9e-7), "temperature"),
    (dict(temperature=1.1e6), "temperature"),
    (dict(values=None), "required"),
    (dict(ids=None), "required"),
    (dict(lse=None), "required"),
    (dict(T=1, V=1 << 20, ld=1 << 20), "workspace"),                       # a row in parts
    (dict(T=1, V=1 << 20, ld=1 << 20, workspace=FAKE, workspace_bytes=16), "workspace"),
    (dict(T=1, V=1 << 20, ld=1 << 20, workspace=FAKE + 8, workspace_bytes=1 << 30), "16-byte"),
])
def test_top_logits_refuses(kw, words):
    refused(top(**kw), words)


def test_top_logits_workspace():
    size = _lib.lib().top_logits_workspace_bytes
    assert size(_lib.DPPO_BF16, 100000, 1000, 8) == 0
    assert size(_lib.DPPO_BF16, 0, 1000, 8) == 0
    assert size(_lib.DPPO_BF16, 1, 1 << 20, 8) > 0
    for bad in ((7, 1, 10, 1), (0, -1, 10, 1), (0, 1, 0, 1), (0, 1, (1 << 28) + 1, 1), (0, 1, 10, 0), (0, 1, 10, 11),
                (0, 1, 1000, 257), (0, 1 << 31, 10, 1)):
        assert size(*bad) == -1


# ---------------------------------------------------------------- distill_loss_fwd_bwd
DISTILL = dict(logits=FAKE, dtype=_lib.DPPO_BF16, T=4, V=1000, ld=1000, values=FAKE, ids=FAKE, k=8, lse=None, mask=None,
               tscale=None, temperature=1.0, scale_mode=0, loss_scale=1.0, kl=FAKE, loss=FAKE, flags=FAKE, stats=FAKE,
               dlogits=None, ld_dlogits=0, stream=None)


def distill(**kw):
    a = {**DISTILL, **kw}
    return _lib.lib().distill_loss_fwd_bwd(*a.values())


def distill_struct(**kw):
    a = {**DISTILL, **kw}
    order = ("logits", "dtype", "T", "V", "ld", "values", "ids", "k", "lse", "mask", "tscale", "kl", "loss", "flags",
             "stats", "dlogits", "ld_dlogits", "stream", "scale_mode", "temperature", "loss_scale")
    return _lib.lib().distill_loss_call(_lib.DISTILL_CALL.pack(*((a[n] or 0) for n in order)))


@pytest.mark.parametrize("call", [distill, distill_struct])
@pytest.mark.parametrize("kw,words", [
    (dict(logits=None), "logits"),
    (dict(logits=FAKE + 1), "aligned"),
    (dict(dtype=7), "dtype"),
    (dict(T=-1), "T"),
    (dict(V=0), "V"),
    (dict(V=(1 << 28) + 1, ld=1 << 29), "V"),
    (dict(ld=999), "stride"),
    (dict(k=0), "k = 0"),
    (dict(k=257), "k = 257"),
    (dict(values=None), "required"),
    (dict(ids=None), "required"),
    (dict(kl=None), "required"),
    (dict(loss=None), "required"),
    (dict(flags=None), "required"),
    (dict(stats=None), "required"),
    (dict(temperature=0.0), "temperature"),
    (dict(temperature=NAN), "temperature"),
    (dict(scale_mode=2), "scale_mode"),
    (dict(scale_mode=-1), "scale_mode"),
    (dict(loss_scale=INF), "loss_scale"),
    (dict(loss_scale=NAN), "loss_scale"),
    (dict(dlogits=1 << 30, ld_dlogits=999), "stride"),
    (dict(dlogits=(1 << 30) + 1, ld_dlogits=1000), "aligned"),
    (dict(dlogits=FAKE + 64, ld_dlogits=1000), "overlaps"),
    (dict(dlogits=FAKE, ld_dlogits=1001), "overlaps"),
])
def test_distill_refuses(call, kw, words):
    refused(call(**kw), words)


def test_struct_calls_refuse_what_32_bits_would_cut():
    refused(distill_struct(k=(1 << 32) + 8), "k = ")
    refused(distill_struct(dtype=1 << 32), "dtype")
    refused(distill_struct(scale_mode=1 << 32), "scale_mode")
    refused(_lib.lib().distill_loss_call(None), "NULL")
    refused(verify_struct(dtype=1 << 32), "dtype")
    refused(_lib.lib().verify_drafts_call(None), "NULL")


# ---------------------------------------------------------------- verify_drafts
VERIFY = dict(target=FAKE, target_seq=5000, target_row=1000, draft=FAKE, draft_seq=4000, draft_row=1000,
              dtype=_lib.DPPO_BF16, B=2, D=4, V=1000, ids=FAKE, num=None, u=FAKE, u_new=FAKE, temperature=1.0,
              accepted=FAKE, tokens=FAKE, logp=FAKE, workspace=FAKE, workspace_bytes=1 << 30, stream=None)


def verify(**kw):
    a = {**VERIFY, **kw}
    return _lib.lib().verify_drafts(*a.values())


def verify_struct(**kw):
    a = {**VERIFY, **kw}
    order = ("target", "target_seq", "target_row", "draft", "draft_seq", "draft_row", "dtype", "B", "D", "V", "ids",
             "num", "u", "u_new", "accepted", "tokens", "logp", "workspace", "workspace_bytes", "stream", "temperature")
    return _lib.lib().verify_drafts_call(_lib.VERIFY_CALL.pack(*((a[n] or 0) for n in order)))


@pytest.mark.parametrize("call", [verify, verify_struct])
@pytest.mark.parametrize("kw,words", [
    (dict(target=None), "target"),
    (dict(target=FAKE + 1), "aligned"),
    (dict(draft=FAKE + 1), "aligned"),
    (dict(dtype=7), "dtype"),
    (dict(B=-1), "B = -1"),
    (dict(B=(1 << 20) + 1), "B = "),
    (dict(D=-1), "D = -1"),
    (dict(D=1025), "D = 1025"),
    (dict(V=0), "V"),
    (dict(V=(1 << 28) + 1), "V"),
    (dict(target_row=999), "stride"),
    (dict(target_seq=999), "stride"),
    (dict(target_seq=0), "stride"),
    (dict(draft_row=999), "stride"),
    (dict(draft_seq=0), "stride"),
    (dict(ids=None), "required"),
    (dict(u=None), "required"),
    (dict(u_new=None), "required"),
    (dict(accepted=None), "required"),
    (dict(tokens=None), "required"),
    (dict(logp=None), "required"),
    (dict(temperature=0.0), "temperature"),
    (dict(temperature=INF), "temperature"),
    (dict(workspace=None), "workspace"),
    (dict(workspace_bytes=100), "workspace"),
    (dict(workspace=FAKE + 4), "16-byte"),
])
def test_verify_refuses(call, kw, words):
    refused(call(**kw), words)


def test_verify_workspace():
    size = _lib.lib().verify_drafts_workspace_bytes
    assert size(_lib.DPPO_BF16, 2, 4, 1000, 1) > 0
    for bad in ((7, 1, 1, 10, 1), (0, -1, 1, 10, 1), (0, (1 << 20) + 1, 1, 10, 1), (0, 1, -1, 10, 1), (0, 1, 1025, 10, 1),
                (0, 1, 1, 0, 1), (0, 1, 1, (1 << 28) + 1, 1)):
        assert size(*bad) == -1


# ---------------------------------------------------------------- the binding
def test_tensors_off_the_gpu_are_refused():
    z = torch.zeros(2, 10)
    rec = (torch.zeros(2, 3), torch.zeros(2, 3, dtype=torch.int32))
    with pytest.raises(ValueError, match="GPU"):
        P.top_logits(z, 3)
    with pytest.raises(ValueError, match="GPU"):
        P.distill_loss_fwd_bwd(z, *rec)
    with pytest.raises(ValueError, match="GPU"):
        P.verify_drafts(z[None], torch.zeros(1, 1, dtype=torch.int64), torch.zeros(1, 1), torch.zeros(1))


@pytest.mark.gpu
def test_binding_refuses():
    dev = "cuda:0"
    z = torch.zeros(4, 10, device=dev)
    v, i = torch.zeros(4, 3, device=dev), torch.zeros(4, 3, dtype=torch.int32, device=dev)
    for bad, err in ((z.half(), TypeError), (z[0], ValueError), (z.t(), ValueError), (z.expand(4, 10)[:, ::2], ValueError)):
        with pytest.raises(err):
            P.top_logits(bad, 3)
        with pytest.raises(err):
            P.distill_loss_fwd_bwd(bad, v, i)
    lazily_negated = torch.complex(z, z).conj().imag
    for call in (lambda t: P.top_logits(t, 3), lambda t: P.distill_loss_fwd_bwd(t, v, i)):
        with pytest.raises(ValueError):
            call(lazily_negated)
    for k in (0, -1, 11, 257, (1 << 32) + 3, -(1 << 32) + 3):
        with pytest.raises(P.DppoError):
            P.top_logits(z, k)
    with pytest.raises(P.DppoError):
        P.top_logits(z[:1].expand(4, 10), 3)              # overlapping rows
    for kw in (dict(teacher_values=v.double()), dict(teacher_values=v[:3]), dict(teacher_values=v[0]),
               dict(teacher_ids=i.long()), dict(teacher_ids=i[:, :2]), dict(teacher_values=v.cpu()),
               dict(teacher_lse=v[:, 0]), dict(loss_mask=torch.ones(4, device=dev)), dict(token_scale=v[:3, 0].contiguous()),
               dict(scale_mode="mean"), dict(dlogits=z.bfloat16()), dict(dlogits=z[:3]),
               dict(dlogits=torch.zeros(10, 4, device=dev).t())):
        with pytest.raises(ValueError):
            P.distill_loss_fwd_bwd(z, **{**dict(teacher_values=v, teacher_ids=i), **kw})
    t = torch.zeros(2, 3, 10, device=dev)
    ok = dict(target_logits=t, draft_ids=torch.zeros(2, 2, dtype=torch.int64, device=dev),
              accept_u=torch.zeros(2, 2, device=dev), sample_u=torch.zeros(2, device=dev))
    assert P.verify_drafts(**ok).tokens.shape == (2, 3)
    for kw in (dict(target_logits=t[0]), dict(target_logits=t[:, :0]), dict(target_logits=t.transpose(1, 2)),
               dict(draft_ids=ok["draft_ids"].int()), dict(draft_ids=ok["draft_ids"][:, :1]), dict(accept_u=t[:, :2, 0]),
               dict(accept_u=ok["accept_u"].double()), dict(sample_u=torch.zeros(3, device=dev)),
               dict(draft_logits=t), dict(draft_logits=t[:, :2].bfloat16()),
               dict(num_drafts=torch.zeros(2, dtype=torch.int64, device=dev)), dict(sample_u=torch.zeros(2))):
        with pytest.raises(ValueError):
            P.verify_drafts(**{**ok, **kw})
    with pytest.raises(TypeError):
        P.verify_drafts(**{**ok, "target_logits": t.half()})
