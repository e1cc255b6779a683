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
