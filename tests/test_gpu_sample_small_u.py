"""sample_tokens for uniform numbers far below a 64-bit step of the total: the tokens in front have so little weight."""
import pytest
import torch

from tests import vocab_ops_ref as ref

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [40, 300, 5000, 9001, 50257])
def test_small_uniform_numbers(gls, V, dtype):
    g = torch.Generator(device="cuda").manual_seed(V)
    x = 2.0 * torch.randn((4, 1, 6, V), generator=g, device="cuda")
    x[..., : V // 2] -= 60.0  # what is in front of the largest logits has 1e-26 of the total
    x[1, ..., : V // 4] -= 20.0
    x[2, ..., V // 2 + 3:] -= 80.0
    x = x.to(dtype)
    u = torch.tensor([1e-35, 1e-30, 1e-27, 1e-25, 1e-18, 1e-12], device="cuda").expand(4, 1, 6).contiguous()
    for kw in (dict(), dict(top_k=V - 1), dict(top_k=V // 2 + V // 4 + 1, top_p=1.0), dict(min_p=1e-37), dict(top_k=V // 2 + V // 4 + 1, top_p=0.9999999, min_p=1e-30)):
        got = gls.sample_tokens(x, u, **kw)
        tokens, lp = ref.sample(x, u, **kw)
        assert torch.equal(got["tokens"].cpu().long(), tokens), (kw, got["tokens"].flatten().tolist(), tokens.flatten().tolist())
        assert bool(((got["logprobs"].cpu().double() - lp).abs() <= ref.SLP + ref.U * lp.abs()).all()), kw
