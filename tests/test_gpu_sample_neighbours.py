"""sample_tokens where neighbouring fp32 logits are tens to thousands of powers of two apart: their weights run out of the
64-bit range within a few steps below the largest logit."""
import pytest
import torch

from tests import vocab_ops_ref as ref

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("V", [64, 3000, 20000])
@pytest.mark.parametrize("exponents", [45.0, 68.9, 95.0, 95.2, 180.0, 334.0, 600.0, 990.0, 1400.0, 1900.0])
def test_steps_below_the_largest_logit(gls, V, exponents):
    """Logits 0 .. 40 steps below the largest, `exponents` powers of two apart (as far as fp32 holds the inverse temperature)."""
    g = torch.Generator(device="cuda").manual_seed(V)
    step = 2.0 ** -17  # of fp32 at 100
    x = torch.where(torch.rand((4, 1, 8, V), generator=g, device="cuda") < 0.5, 100.0 - 3.0 * torch.rand((4, 1, 8, V), generator=g, device="cuda"),
                    100.0 - step * torch.randint(0, 41, (4, 1, 8, V), generator=g, device="cuda"))
    x[1] += step * (x[1] < 100.0)  # nothing at one step
    u = torch.rand((4, 1, 8), generator=g, device="cuda")
    it = ref.f32(exponents / step / 1.4426950408889634)
    few, many = min(400, V - 1), min(2500, V - 1)
    for kw in (dict(top_k=30), dict(top_k=few), dict(top_k=40, top_p=0.9), dict(top_k=many, top_p=0.9), dict(min_p=0.1), dict(min_p=1e-35)):
        got = gls.sample_tokens(x, u, inv_temp=it, **kw)
        tokens, lp = ref.sample(x, u, inv_temp=it, **kw)
        assert torch.equal(got["tokens"].cpu().long(), tokens), kw
        assert bool(((got["logprobs"].cpu().double() - lp).abs() <= ref.SLP + ref.U * lp.abs()).all()), kw
