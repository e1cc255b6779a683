"""Arguments that the log-probability and embedding entry points refuse.  Every call here is answered on
the host before anything is enqueued, so no GPU is needed: the pointers are made up and never read.
Where a GPU is present the tests are skipped, so that no kernel can ever see one of them."""
import ctypes as C

import pytest
import torch

import paper_2506_05632_b200 as gls
from paper_2506_05632_b200 import binding

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="made-up pointers: only where no kernel can start")

OK, INVALID, UNSUPPORTED, MISALIGNED, WORKSPACE = 0, 1, 2, 3, 4
P = 0x10000000  # an aligned address


def _rows(dtype=1, data=P, sb=1000, sk=1000, sj=1000):
    return binding._Rows(data, dtype, sb, sk, sj)


def _logprobs(**kw):
    a = dict(rows=_rows(), B=2, K=2, J=2, V=1000, it=1.0, per=None, tokens=P, G=1, M=5, lp=P, lse=P, tail=None,
             ent=P, ids=P, tlp=P)
    a.update(kw)
    return gls.load().gls_token_logprobs(C.byref(a["rows"]), a["B"], a["K"], a["J"], a["V"], a["it"], a["per"],
                                         a["tokens"], a["G"], a["M"], a["lp"], a["lse"], a["tail"], a["ent"],
                                         a["ids"], a["tlp"], None, None)


@pytest.mark.parametrize("kw,status", [
    (dict(B=0), INVALID), (dict(K=0), INVALID), (dict(K=65), INVALID), (dict(J=-1), INVALID),
    (dict(V=0), INVALID), (dict(V=1 << 31), INVALID), (dict(G=-1), INVALID), (dict(G=65), INVALID),
    (dict(M=-1), INVALID), (dict(M=257), INVALID), (dict(tokens=None), INVALID), (dict(lp=None), INVALID),
    (dict(lse=None), INVALID), (dict(ids=None), INVALID), (dict(tlp=None), INVALID),
    (dict(it=0.0), INVALID), (dict(it=-1.0), INVALID), (dict(it=float("nan")), INVALID),
    (dict(it=float("inf")), INVALID), (dict(it=1e-30), UNSUPPORTED), (dict(it=1e30), UNSUPPORTED),
    (dict(rows=_rows(data=None)), INVALID), (dict(rows=_rows(dtype=2)), UNSUPPORTED),
    (dict(rows=_rows(data=P + 1)), MISALIGNED), (dict(rows=_rows(dtype=0, data=P + 2)), MISALIGNED),
])
def test_logprobs_refusals(kw, status):
    assert _logprobs(**kw) == status


def test_logprobs_per_draft_temperatures_are_checked():
    bad = (C.c_float * 2)(1.0, 0.0)
    assert _logprobs(per=C.cast(bad, C.c_void_p)) == INVALID


def _emitted(**kw):
    a = dict(rows=_rows(), B=2, K=2, L=2, V=1000, it=1.0, tokens=P, accept=P, flags=0, M=5, lp=P, lse=P, ent=P,
             ids=P, tlp=P)
    a.update(kw)
    return gls.load().gls_emitted_logprobs(C.byref(a["rows"]), a["B"], a["K"], a["L"], a["V"], a["it"], a["tokens"],
                                           a["accept"], a["flags"], a["M"], a["lp"], a["lse"], a["ent"], a["ids"],
                                           a["tlp"], None, None)


@pytest.mark.parametrize("kw,status", [
    (dict(L=-1), INVALID), (dict(L=0, flags=2), INVALID), (dict(tokens=None), INVALID),
    (dict(accept=None), INVALID), (dict(flags=4), INVALID), (dict(flags=64), INVALID), (dict(lp=None), INVALID),
    (dict(M=300), INVALID), (dict(K=65), INVALID), (dict(it=0.0), INVALID),
])
def test_emitted_refusals(kw, status):
    assert _emitted(**kw) == status


def _backward(**kw):
    a = dict(rows=_rows(), B=2, K=2, J=2, V=1000, it=1.0, tokens=P, G=1, ids=P, M=5, lse=P, tail=None, ent=P,
             glp=P, glse=P, gent=P, gtop=P, out=_rows(data=2 * P))
    a.update(kw)
    return gls.load().gls_token_logprobs_backward(C.byref(a["rows"]), a["B"], a["K"], a["J"], a["V"], a["it"], None,
                                                  a["tokens"], a["G"], a["ids"], a["M"], a["lse"], a["tail"],
                                                  a["ent"], a["glp"], a["glse"], a["gent"], a["gtop"],
                                                  C.byref(a["out"]), None)


@pytest.mark.parametrize("kw,status", [
    (dict(lse=None), INVALID), (dict(tokens=None), INVALID), (dict(ids=None), INVALID), (dict(ent=None), INVALID),
    (dict(G=65), INVALID), (dict(M=257), INVALID), (dict(V=0), INVALID), (dict(it=float("nan")), INVALID),
    (dict(out=_rows(data=P)), INVALID),                      # the logits' own memory
    (dict(out=_rows(data=2 * P, sb=0)), INVALID), (dict(out=_rows(data=2 * P, sk=0)), INVALID),
    (dict(out=_rows(data=2 * P, sj=0)), INVALID),            # several rows in one place
    (dict(out=_rows(data=2 * P, dtype=0)), UNSUPPORTED), (dict(out=_rows(data=2 * P + 1)), MISALIGNED),
    (dict(out=_rows(data=None)), INVALID), (dict(it=1e25), UNSUPPORTED),
])
def test_backward_refusals(kw, status):
    assert _backward(**kw) == status


def _embed(**kw):
    a = dict(table=P, dtype=1, ts=64, V=100, D=64, tokens=P, N=10, scale=1.0, out=P, os=64)
    a.update(kw)
    return gls.load().gls_embed_tokens(a["table"], a["dtype"], a["ts"], a["V"], a["D"], a["tokens"], a["N"],
                                       a["scale"], a["out"], a["os"], None, None)


@pytest.mark.parametrize("kw,status", [
    (dict(table=None), INVALID), (dict(tokens=None), INVALID), (dict(out=None), INVALID), (dict(V=0), INVALID),
    (dict(D=0), INVALID), (dict(N=-1), INVALID), (dict(N=1 << 31), INVALID), (dict(ts=63), INVALID),
    (dict(os=0), INVALID), (dict(scale=float("nan")), INVALID), (dict(scale=float("inf")), INVALID),
    (dict(dtype=2), UNSUPPORTED), (dict(table=P + 1), MISALIGNED), (dict(out=P + 2, dtype=0), MISALIGNED),
    (dict(N=0), OK), (dict(N=0, table=None, tokens=None, out=None), OK),
])
def test_embed_refusals(kw, status):
    assert _embed(**kw) == status


def _embed_backward(**kw):
    a = dict(g=P, dtype=1, gs=64, tokens=P, N=10, V=100, D=64, scale=1.0, table=P, gdtype=1, ts=64, flags=0, ws=P,
             n=1 << 30)
    a.update(kw)
    return gls.load().gls_embed_tokens_backward(a["g"], a["dtype"], a["gs"], a["tokens"], a["N"], a["V"], a["D"],
                                                a["scale"], a["table"], a["gdtype"], a["ts"], a["flags"], a["ws"],
                                                a["n"], None, None)


@pytest.mark.parametrize("kw,status", [
    (dict(g=None), INVALID), (dict(tokens=None), INVALID), (dict(table=None), INVALID), (dict(V=0), INVALID),
    (dict(D=-1), INVALID), (dict(N=1 << 30), INVALID), (dict(gs=10), INVALID), (dict(ts=0), INVALID),
    (dict(flags=2), INVALID), (dict(scale=float("inf")), INVALID), (dict(dtype=3), UNSUPPORTED),
    (dict(dtype=0, gdtype=1), UNSUPPORTED),                  # fp32 sums into a bf16 table
    (dict(g=P + 1), MISALIGNED), (dict(table=P + 1), MISALIGNED), (dict(ws=None), WORKSPACE),
    (dict(n=100), WORKSPACE), (dict(ws=P + 8), MISALIGNED), (dict(N=0, flags=1), OK),
])
def test_embed_backward_refusals(kw, status):
    assert _embed_backward(**kw) == status


def test_workspace_sizes():
    small = gls.embed_tokens_backward_workspace_bytes(10, 100, 64)
    assert 0 < small < gls.embed_tokens_backward_workspace_bytes(100000, 100, 64)
    assert gls.embed_tokens_backward_workspace_bytes(10, 0, 64) == 0


def test_host_tensors_are_refused():
    x, t = torch.zeros(1, 1, 1, 8), torch.zeros(1, 1, 1, dtype=torch.int32)
    with pytest.raises(gls.GlsError):
        gls.token_logprobs(x, t)
    with pytest.raises(gls.GlsError):
        gls.emitted_logprobs(x, t[0], None)
    with pytest.raises(gls.GlsError):
        gls.token_logprobs_backward(x, t, torch.zeros(1, 1, 1))
    with pytest.raises(gls.GlsError):
        gls.embed_tokens(torch.zeros(4, 8), t)
    with pytest.raises(gls.GlsError):
        gls.embed_tokens_backward(torch.zeros(1, 1, 1, 8), t, 4)
