"""What the operators next to the sampler do with tensors that ask for a derivative they do not have."""
import pytest
import torch
from torch.autograd import forward_ad

import paper_2506_05632_b200 as gls

X, TABLE = torch.zeros(1, 2, 3, 50), torch.zeros(9, 4)
TOK = torch.zeros(1, 2, 3, dtype=torch.int32)
ROWS = torch.zeros(1, 2, 3)


def _dual(t, requires_grad):
    return forward_ad.make_dual(t.clone().requires_grad_(requires_grad), torch.ones_like(t))


@pytest.mark.parametrize("requires_grad", [False, True])
@pytest.mark.parametrize("call", [
    lambda d: gls.token_logprobs(d(X), TOK),
    lambda d: gls.token_logprobs(d(X), TOK, out={}),
    lambda d: gls.emitted_logprobs(d(X), TOK[:, 0], torch.zeros(1, 2, 2, dtype=torch.uint8)),
    lambda d: gls.embed_tokens(d(TABLE), TOK),
    lambda d: gls.token_logprobs_backward(X, TOK, ROWS, grad_lse=d(ROWS)),
    lambda d: gls.token_logprobs_backward(d(X), TOK, ROWS, grad_lse=ROWS),
    lambda d: gls.embed_tokens_backward(d(TABLE[:6].view(1, 2, 3, 4)), TOK, 9),
])
def test_tangents_are_refused(call, requires_grad):
    """A dual tensor's result would come back without its tangent."""
    with forward_ad.dual_level():
        with pytest.raises(gls.GlsError, match="forward-mode"):
            call(lambda t: _dual(t, requires_grad))
        with torch.no_grad(), pytest.raises(gls.GlsError, match="forward-mode"):
            call(lambda t: _dual(t, requires_grad))
        with pytest.raises(gls.GlsError) as e:  # the level alone changes nothing: these have no tangent
            call(lambda t: t)
        assert "forward-mode" not in str(e.value)


def test_emitted_logprobs_of_logits_that_require_a_gradient():
    """They would come back without a history and drop out of a loss."""
    x = X.clone().requires_grad_()
    args = TOK[:, 0], torch.zeros(1, 2, 2, dtype=torch.uint8)
    with pytest.raises(gls.GlsError, match="no gradient"):
        gls.emitted_logprobs(x, *args)
    for y, grad in ((x.detach(), True), (x, False)):  # on the way to the kernel, which there is not here
        with torch.set_grad_enabled(grad), pytest.raises(gls.GlsError, match="device tensors"):
            gls.emitted_logprobs(y, *args)


@pytest.mark.gpu
def test_a_step_on_logits_that_require_a_gradient(gls):
    """The serving step reports on them all the same: its results carry no gradient."""
    from paper_2506_05632_b200 import pipeline

    t = torch.randn((3, 2, 3, 600), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    out = []
    for x in (t, t.clone().requires_grad_()):
        buf = pipeline.StepBuffers(3, 2, 2, 600, top=4)
        pipeline.spec_step(x[:, :, :2], x, buf, seed=3)
        out.append(buf.answers)
    for n in out[0]:
        assert torch.equal(out[0][n], out[1][n]) and not out[1][n].requires_grad


@pytest.mark.gpu
def test_tokens_overwritten_before_the_backward_pass(gls):
    """A backward pass whose tokens a later call has written over would return another batch's gradient."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((2, 3, 2, 700), generator=gen, device="cuda")
    table = torch.randn((700, 16), generator=gen, device="cuda", requires_grad=True)
    head = torch.randn((16, 700), generator=gen, device="cuda", requires_grad=True)
    for late in (False, True):
        tok, _ = gls.draft_sample(x, seed=1, out_tokens=torch.empty((2, 3, 2), dtype=torch.int32, device="cuda"))
        h = gls.embed_tokens(table, tok)
        lp = gls.token_logprobs(h @ head, tok)["logprobs"]
        if late:
            gls.draft_sample(x, seed=2, out_tokens=tok)
            with pytest.raises(RuntimeError, match="modified by an inplace operation"):
                lp.sum().backward()
            with pytest.raises(RuntimeError, match="modified by an inplace operation"):
                h.sum().backward()
        else:
            lp.sum().backward()
            assert table.grad is not None


@pytest.mark.gpu
def test_every_written_tensor_counts_as_changed(gls):
    from paper_2506_05632_b200 import pipeline

    B, K, L, V, D = 2, 3, 2, 640, 8
    gen = torch.Generator(device="cuda").manual_seed(2)
    t = torch.randn((B, K, L + 1, V), generator=gen, device="cuda")
    d = t[:, :, :L]
    tok, sc = gls.draft_sample(d, seed=1)
    out = gls.target_sample_verify(t, tok, seed=1)
    ans = gls.emitted_logprobs(t, out["tokens"], out["accept"], top=2)
    lp = gls.token_logprobs(t, None, top=2)
    table = torch.randn((V, D), generator=gen, device="cuda")
    rows = gls.embed_tokens(table, out["tokens"])
    enc, dec = t[:, 0, 0].contiguous(), t[:, :, 0].contiguous()
    sel = gls.compress_select(enc, dec, seed=1)
    u, a, s = (torch.randn(n, generator=gen, device="cuda") for n in ((V, 4), (B, 4), (B, K, 4)))
    gau = gls.compress_gaussian(u, a, s, seed=1)
    space = torch.empty(gls.topm_workspace_bytes(B, K, L + 1, 5), dtype=torch.uint8, device="cuda")
    host = torch.zeros((4, 10)).pin_memory()
    dev = torch.zeros((4, 10), device="cuda")
    grad = torch.empty_like(t)
    calls = [
        (lambda: gls.draft_sample(d, seed=1, out_tokens=tok, out_scores=sc), [tok, sc]),
        (lambda: gls.draft_sample_static(d, tok, sc, seed=1), [tok, sc]),
        (lambda: gls.target_sample_verify(t, tok, seed=1, out=out), list(out.values())),
        (lambda: gls.draft_verify(d, t, seed=1, out_draft_tokens=tok, out_draft_scores=sc, out=out), [tok, sc, *out.values()]),
        (lambda: gls.draft_sample_topm(d, 5, seed=1, workspace=space), [space]),
        (lambda: gls.target_sample_verify_topm(t, tok, 5, seed=1, workspace=space), [space]),
        (lambda: gls.compress_select(enc, dec, seed=1, out=sel), list(sel.values())),
        (lambda: gls.compress_gaussian(u, a, s, seed=1, out=gau), list(gau.values())),
        (lambda: gls.copy_rows_to_device(dev, host), [dev]),
        (lambda: gls.emitted_logprobs(t, out["tokens"], out["accept"], top=2, out=ans), list(ans.values())),
        (lambda: gls.token_logprobs(t, None, top=2, out=lp), list(lp.values())),
        (lambda: gls.token_logprobs_backward(t, None, lp["lse"], grad_lse=lp["lse"], grad_logits=grad), [grad]),
        (lambda: gls.embed_tokens(table, out["tokens"], out=rows), [rows]),
        (lambda: gls.embed_tokens_backward(rows, out["tokens"], V, grad_table=table, accumulate=True), [table]),
    ]
    for n, (call, written) in enumerate(calls):
        before = [w._version for w in written]
        call()
        assert all(w._version > b for w, b in zip(written, before)), n
    buf = pipeline.StepBuffers(B, K, L, V, top=2, table=table)
    step = pipeline.GraphedStep(d, t, buf, seed=1)
    written = [buf.draft_tokens, buf.draft_scores, buf.inputs, *buf.out.values(), *buf.answers.values()]
    before = [w._version for w in written]
    step.replay()
    assert all(w._version > b for w, b in zip(written, before))
    with torch.inference_mode():  # tensors that keep no count
        tok2 = torch.empty_like(tok)
        gls.draft_sample(d.clone(), seed=1, out_tokens=tok2)
    torch.cuda.synchronize()
    assert torch.equal(tok2, tok)
