"""sample_tokens where top-p's border falls exactly between tokens of the largest logit: shares that fp32 holds of numbers
of equal weights that they divide."""
import pytest
import torch

from tests import vocab_ops_ref as ref

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V,n", [(40, 40), (4000, 4), (4000, 96), (4000, 3600), (20000, 8), (20000, 1000), (20000, 16000)])
def test_exact_shares_of_the_largest(gls, V, n, dtype):
    """n tokens of one logit and others that have no weight beside them: the first p n of them stay, not one more."""
    g = torch.Generator(device="cuda").manual_seed(V + n)
    for value, it in ((10.3, 0.7), (-7.1, 1.0), (14.7, 1.0), (1234.5, 1.3), (0.013, 900.0), (91.3, 1000.0)):
        x = torch.full((4, 1, 4, V), value - 150.0 / it, device="cuda")
        x.scatter_(-1, torch.rand((4, 1, 4, V), generator=g, device="cuda").argsort(-1)[..., :n], value)
        x = x.to(dtype)
        u = torch.rand((4, 1, 4), generator=g, device="cuda")
        u[..., -1] = 1.0  # the last of those that stay
        for kw in (dict(top_p=0.5), dict(top_p=0.75), dict(top_k=V - 1, top_p=0.5), dict(top_k=(n + 1) // 2, top_p=0.5), dict(top_p=0.25, min_p=0.1)):
            got = gls.sample_tokens(x, u, inv_temp=ref.f32(it), **kw)
            tokens, lp = ref.sample(x, u, inv_temp=ref.f32(it), **kw)
            assert torch.equal(got["tokens"].cpu().long(), tokens), (value, it, kw, got["tokens"].cpu().flatten().tolist(), tokens.flatten().tolist())
            assert bool(((got["logprobs"].cpu().double() - lp).abs() <= ref.SLP + ref.U * lp.abs()).all()), (value, it, kw)
