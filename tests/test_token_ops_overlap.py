"""Embedding calls whose output would lie in the memory that they read are refused; columns of one buffer
that do not meet are not."""
import pytest
import torch

from tests.test_token_ops_refusals import INVALID, P, _embed, _embed_backward

no_gpu = pytest.mark.skipif(torch.cuda.is_available(), reason="made-up pointers: only where no kernel can start")
BF = 2  # bytes of an element


@no_gpu
@pytest.mark.parametrize("kw", [
    dict(out=P),                                              # the table itself
    dict(out=P + 99 * 64 * BF),                               # its last row
    dict(out=P - 9 * 64 * BF),                                # the last output is its first row
    dict(out=P + 64, ts=100, os=100),                         # columns 32 .. 96 of the table's buffer
    dict(out=P + 80 * BF, ts=100, os=100),                    # columns 80 .. 144 of rows 100 apart
    dict(out=P + 128, ts=200, os=400),                        # other distances between rows
    dict(out=P + 63 * BF, V=1, ts=0),                         # one row of either
    dict(out=P + 63 * BF, V=1, ts=0, N=1, os=0),
    dict(out=P + 99 * 64 * BF, N=1, os=0), dict(out=P, ts=1 << 60, os=1 << 60),
])
def test_lookup_into_its_table(kw):
    assert _embed(**kw) == INVALID


@no_gpu
@pytest.mark.parametrize("kw", [
    dict(table=P, g=P, ws=9 * P), dict(table=P + 64, g=P, gs=100, ts=100, ws=9 * P),
    dict(table=P + 9 * 64 * BF, g=P, ws=9 * P), dict(table=P - 99 * 64 * 4, g=P, gdtype=0, ws=9 * P, flags=1),
    dict(table=P, g=P + 64, gs=64, ts=64, gdtype=0, ws=9 * P), dict(table=P, g=P + 100 * 64 * BF - 2, N=1, gs=0, ws=9 * P),
])
def test_gradient_into_what_it_reads(kw):
    assert _embed_backward(**kw) == INVALID


@pytest.mark.gpu
def test_columns_of_one_buffer(gls):
    gen = torch.Generator(device="cuda").manual_seed(1)
    buf = torch.randn((50, 130), generator=gen, device="cuda")
    tok = torch.randint(50, (50,), generator=gen, device="cuda").to(torch.int32)
    table = buf[:, 3:67]
    want = table[tok.long()]
    for out in (buf[:, 66:130], buf[:, 1:65], buf[:40, 3:67], buf[49:50, 3:67]):
        with pytest.raises(gls.GlsError):
            gls.embed_tokens(table, tok[:out.shape[0]].contiguous(), out=out)
    before = buf.clone()
    side = torch.randn((50, 140), generator=gen, device="cuda")
    side[:, :64] = table
    left, right = side[:, :64], side[:, 64:128]
    assert torch.equal(gls.embed_tokens(left, tok, out=right), want) and torch.equal(left, table)
    assert torch.equal(buf, before)
    one = side[49:50, 128:140]  # behind the last row of the left columns
    gls.embed_tokens(side[:, :12], tok[:1], out=one)
    assert torch.equal(one, side[:, :12][tok[:1].long()])
    grad = gls.embed_tokens_backward(left, tok, 50)
    gls.embed_tokens_backward(left, tok, 50, grad_table=right)
    assert torch.equal(grad, right) and torch.equal(left, table)
    with pytest.raises(gls.GlsError):
        gls.embed_tokens_backward(left, tok, 50, grad_table=side[:, 63:127])
