"""Arguments that the sampling and 4-bit entry points refuse.  Every call here is answered on the host before anything is
enqueued, so no GPU is needed: the pointers are made up and never read.  Where a GPU is present the tests are
skipped, so that no kernel can ever see one of them."""
import ctypes as C

import pytest
import torch

import paper_2506_05632_b200 as gls
from paper_2506_05632_b200 import binding

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="made-up pointers: only where no kernel can start")

OK, INVALID, UNSUPPORTED, MISALIGNED, WORKSPACE = 0, 1, 2, 3, 4
P = 0x10000000  # an aligned address
INF, NAN = float("inf"), float("nan")


def _sample(**kw):
    a = dict(rows=binding._Rows(P, 1, 1000, 1000, 1000), B=2, K=2, J=2, V=1000, it=1.0, k=0, p=1.0, m=0.0, itr=None, pr=None,
             mr=None, u=P, tok=P, lp=P, s=True)
    a.update(kw)
    s = binding._Sampling(a["it"], a["k"], a["p"], a["m"], a["itr"], None, a["pr"], a["mr"])
    return gls.load().gls_sample_tokens(C.byref(a["rows"]) if a["rows"] else None, a["B"], a["K"], a["J"], a["V"],
                                        C.byref(s) if a["s"] else None, a["u"], a["tok"], a["lp"], None, None)


@pytest.mark.parametrize("kw,status", [
    (dict(B=0), INVALID), (dict(K=0), INVALID), (dict(K=65), INVALID), (dict(J=0), INVALID), (dict(V=0), INVALID),
    (dict(V=1 << 31), INVALID), (dict(B=1 << 25), INVALID), (dict(rows=None), INVALID), (dict(s=False), INVALID),
    (dict(u=None), INVALID), (dict(tok=None), INVALID), (dict(rows=binding._Rows(None, 1, 1, 1, 1)), INVALID),
    (dict(rows=binding._Rows(P, 2, 1, 1, 1)), UNSUPPORTED), (dict(rows=binding._Rows(P + 1, 1, 1, 1, 1)), MISALIGNED),
    (dict(rows=binding._Rows(P + 2, 0, 1, 1, 1)), MISALIGNED),
    (dict(it=0.0), INVALID), (dict(it=-1.0), INVALID), (dict(it=NAN), INVALID), (dict(it=-INF), INVALID),
    (dict(it=1e-30), UNSUPPORTED), (dict(it=1e30), UNSUPPORTED), (dict(p=0.0), INVALID), (dict(p=NAN), INVALID),
    (dict(p=-1.0), INVALID), (dict(m=-0.1), INVALID), (dict(m=1.1), INVALID), (dict(m=NAN), INVALID),
    (dict(it=0.0, itr=P, p=0.0), INVALID),
])
def test_sample_refusals(kw, status):
    assert _sample(**kw) == status


def _table(**kw):
    a = dict(codes=P, cs=64, scales=2 * P, sd=1, ss=4, zeros=3 * P, zs=4, V=50, D=128, group=32)
    a.update(kw)
    return binding._Int4(a["codes"], a["cs"], a["scales"], a["sd"], a["ss"], a["zeros"], a["zs"], a["V"], a["D"], a["group"])


BAD_TABLES = [
    (dict(codes=None), INVALID), (dict(scales=None), INVALID), (dict(V=0), INVALID), (dict(V=1 << 31), INVALID),
    (dict(D=0), INVALID), (dict(cs=48), INVALID), (dict(ss=3), INVALID), (dict(zs=3), INVALID), (dict(group=16), UNSUPPORTED),
    (dict(group=100), UNSUPPORTED), (dict(sd=2), UNSUPPORTED), (dict(D=32769, cs=1 << 15, ss=2000, zs=2000), UNSUPPORTED),
    (dict(codes=P + 8), MISALIGNED), (dict(cs=72), MISALIGNED), (dict(scales=2 * P + 1), MISALIGNED),
    (dict(scales=2 * P + 2, sd=0), MISALIGNED),
]


@pytest.mark.parametrize("kw,status", BAD_TABLES)
def test_bad_tables(kw, status):
    L, t = gls.load(), _table(**kw)
    assert L.gls_head_logits(5 * P, 1, 128, 3, C.byref(t), 6 * P, 1, 50, None, 0, None) == status
    assert L.gls_quantize_table(5 * P, 1, 128, C.byref(t), None) == status
    assert L.gls_embed_tokens_int4(C.byref(t), 7 * P, 3, 1.0, 6 * P, 1, 128, None, None) == status


def _head(**kw):
    a = dict(x=5 * P, xd=1, xs=128, N=3, out=6 * P, od=1, os=50, t=_table(), ws=None, n=0)
    a.update(kw)
    return gls.load().gls_head_logits(a["x"], a["xd"], a["xs"], a["N"], C.byref(a["t"]) if a["t"] else None, a["out"], a["od"], a["os"], a["ws"], a["n"],
                                      None)


@pytest.mark.parametrize("kw,status", [
    (dict(t=None), INVALID), (dict(x=None), INVALID), (dict(out=None), INVALID), (dict(N=-1), INVALID), (dict(N=65536), INVALID),
    (dict(xs=127), INVALID), (dict(os=49), INVALID), (dict(xd=2), UNSUPPORTED), (dict(od=-1), UNSUPPORTED),
    (dict(x=5 * P + 1), MISALIGNED), (dict(out=6 * P + 2, od=0), MISALIGNED), (dict(out=5 * P), INVALID), (dict(out=5 * P + 256), INVALID),
    (dict(out=P + 64), INVALID), (dict(out=2 * P - 100), INVALID), (dict(out=3 * P), INVALID), (dict(N=0), OK),
    (dict(N=0, x=None, out=None), OK), (dict(N=9), WORKSPACE), (dict(N=9, ws=8 * P, n=100), WORKSPACE),
    (dict(N=9, ws=8 * P + 8, n=1 << 20), MISALIGNED), (dict(N=9, ws=6 * P + 64, n=1 << 20), INVALID),
])
def test_head_refusals(kw, status):
    assert _head(**kw) == status


def _embed(**kw):
    a = dict(tok=7 * P, N=3, scale=1.0, out=6 * P, od=1, os=128, t=_table())
    a.update(kw)
    return gls.load().gls_embed_tokens_int4(C.byref(a["t"]) if a["t"] else None, a["tok"], a["N"], a["scale"], a["out"], a["od"], a["os"], None, None)


@pytest.mark.parametrize("kw,status", [
    (dict(t=None), INVALID), (dict(tok=None), INVALID), (dict(out=None), INVALID), (dict(N=-1), INVALID), (dict(N=1 << 31), INVALID),
    (dict(os=127), INVALID), (dict(scale=NAN), INVALID), (dict(scale=INF), INVALID), (dict(od=3), UNSUPPORTED),
    (dict(out=6 * P + 1), MISALIGNED), (dict(out=7 * P - 100, os=128), INVALID), (dict(out=P), INVALID), (dict(out=2 * P), INVALID),
    (dict(N=0), OK), (dict(N=0, tok=None, out=None), OK),
])
def test_embed_refusals(kw, status):
    assert _embed(**kw) == status


@pytest.mark.parametrize("a,status", [
    ((None, 1, 128), INVALID), ((5 * P, 1, 127), INVALID), ((5 * P, 2, 128), UNSUPPORTED), ((5 * P + 1, 1, 128), MISALIGNED),
    ((P, 1, 128), INVALID), ((2 * P, 1, 128), INVALID), ((3 * P + 2, 1, 128), INVALID),
])
def test_quantize_refusals(a, status):
    assert gls.load().gls_quantize_table(*a, C.byref(_table()), None) == status


def test_host_tensors_are_refused():
    x, u = torch.zeros(1, 1, 1, 8), torch.zeros(1, 1, 1)
    t = gls.Int4Table(torch.zeros((4, 16), dtype=torch.uint8), torch.ones((4, 1)), None, 8, 32)
    with pytest.raises(gls.GlsError):
        gls.sample_tokens(x, u)
    with pytest.raises(gls.GlsError):
        gls.head_logits(torch.zeros(2, 8), t)
    with pytest.raises(gls.GlsError):
        gls.embed_tokens_int4(t, torch.zeros(2, dtype=torch.int32))
    with pytest.raises(gls.GlsError):
        gls.quantize_table(torch.zeros(4, 8))
    for call in (lambda: gls.sample_tokens(x.requires_grad_(), u), lambda: gls.head_logits(torch.zeros(2, 8, requires_grad=True), t),
                 lambda: gls.quantize_table(torch.zeros(4, 8, requires_grad=True))):
        with pytest.raises(gls.GlsError, match="no gradient"):
            call()


def test_workspace_sizes():
    f = gls.head_logits_workspace_bytes
    assert f(8, 4096, torch.bfloat16) == 0 and f(9, 4096, torch.bfloat16) == 16 * 4096 * 2
    assert f(64, 4000, torch.float32) == 3 * 64 * 4096 * 2 and f(65, 100, torch.bfloat16) == 2 * 48 * 128 * 2
    assert f(9, 32769, torch.bfloat16) == 0 and f(9, 0, torch.bfloat16) == 0


@pytest.mark.parametrize("ws", [5 * P, 5 * P + 1024, P, 2 * P, 3 * P])
def test_workspace_that_meets_an_input(ws):
    """Hidden states and the table are read after the workspace has been written."""
    assert _head(N=9, ws=ws, n=1 << 20) == INVALID


@pytest.mark.parametrize("k,value", [(5, 5), (0, 0), (-7, -1), (2 ** 31 - 1, 2 ** 31 - 1), (2 ** 31, 2 ** 31 - 1), (2 ** 40 + 5, 2 ** 31 - 1),
                                     (-2 ** 40 + 5, -1), (7.0, 7), (True, 1)])
def test_top_k_beyond_32_bits(k, value):
    s = binding._Sampling()
    binding._setting(s, "top_k", k, torch.int32, (1, 1, 1), 0)
    assert s.top_k == value


@pytest.mark.parametrize("k", [0.5, 50.9, NAN, INF])
def test_top_k_that_is_no_whole_number(k):
    with pytest.raises(gls.GlsError, match="whole number"):
        binding._setting(binding._Sampling(), "top_k", k, torch.int32, (1, 1, 1), 0)


@pytest.mark.parametrize("name", ["inv_temp", "top_p", "min_p"])
def test_settings_that_want_a_gradient(name):
    with pytest.raises(gls.GlsError, match="no gradient"):
        gls.sample_tokens(torch.zeros(1, 1, 1, 8), torch.zeros(1, 1, 1), **{name: torch.ones(1, requires_grad=True)})
