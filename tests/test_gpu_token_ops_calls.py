"""Calls of the operators next to the sampler that their other tests do not make."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_an_argument_without_a_truth_value(gls, monkeypatch):
    """want_entropy that is neither true nor false: the same error by either way of a call."""
    x = torch.zeros((1, 1, 2, 40), device="cuda")
    tok = torch.zeros((1, 1, 2), dtype=torch.int32, device="cuda")
    both = torch.ones(2)
    errors = []
    for stand_in in (False, True):
        if stand_in:
            monkeypatch.setattr(gls.binding, "_calls", gls.binding._GeneralWay())
        for call in (lambda: gls.token_logprobs(x, tok, want_entropy=both),
                     lambda: gls.emitted_logprobs(x[:, :, :1], tok[:, 0, :1], None, want_entropy=both)):
            with pytest.raises(RuntimeError) as e:
                call()
            errors.append((e.type, str(e.value)))
            assert gls.token_logprobs(x, tok)["entropy"].shape == (1, 1, 2)
    assert errors[:2] == errors[2:]
