"""sample_tokens over numbers of rows on either side of every change of CTA size: tokens of a large call equal those of the same
rows in small ones, and a part of them the 64-bit form."""
import math

import pytest
import torch

from tests import vocab_ops_ref as ref

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [1000, 8192, 8193, 30000])
def test_sizes_of_ctas(gls, V, dtype):
    most = 1200
    g = torch.Generator(device="cuda").manual_seed(V)
    x = (3.0 * torch.randn((most, 1, 1, V), generator=g, device="cuda")).to(dtype)
    x[::7] *= 0.1
    u = torch.rand((most, 1, 1), generator=g, device="cuda")
    own = dict(inv_temp=torch.tensor([1.0, 0.5, math.inf, 1.7], device="cuda").repeat(most // 4),
               top_k=torch.tensor([0, 50, 0, 0, 300], dtype=torch.int32, device="cuda").repeat(most // 5),
               top_p=torch.tensor([0.9, 1.0, 0.5], device="cuda").repeat(most // 3))
    for kw in (dict(), dict(top_k=1), dict(top_k=50, top_p=0.9), dict(top_k=600), dict(top_p=0.9), dict(min_p=0.05), own):
        def call(lo, hi):
            return gls.sample_tokens(x[lo:hi], u[lo:hi], **{k: v[lo:hi] if isinstance(v, torch.Tensor) else v for k, v in kw.items()})
        parts = torch.cat([call(i, i + 40)["tokens"] for i in range(0, most, 40)])
        tokens, lp = ref.sample(x[:40], u[:40], **{k: v[:40] if isinstance(v, torch.Tensor) else v for k, v in kw.items()})
        assert torch.equal(parts[:40].cpu().long(), tokens), kw.keys()
        for rows in (100, 148, 149, 200, 592, 593, 700, most):
            got = call(0, rows)
            assert torch.equal(got["tokens"], parts[:rows]), (kw.keys(), rows, int((got["tokens"] != parts[:rows]).sum()))
            off = (got["logprobs"][:40].cpu().double() - lp).abs()
            assert bool((off <= ref.SLP + ref.U * lp.abs()).all()), (kw.keys(), rows)
