"""sample_tokens with a top-k of more tokens than the first bound leaves: the bound is lowered until k tokens reach it, whatever the
logits' sign and spacing, and rows that do not have k tokens end as well."""
import math

import pytest
import torch

from tests import vocab_ops_ref as ref

pytestmark = pytest.mark.gpu


def _check(gls, x, u, **kw):
    got = gls.sample_tokens(x, u, **kw)
    torch.cuda.synchronize()
    tokens, lp = ref.sample(x, u, **kw)
    assert torch.equal(got["tokens"].cpu().long(), tokens), kw
    assert bool(((got["logprobs"].cpu().double() - lp).abs() <= ref.SLP + ref.U * lp.abs()).all()), kw


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("offset", [0.0, -10.0, -77.7, -300.0, 10.3, -1e-3, -1e30])
def test_logits_close_to_one_another(gls, offset, dtype):
    """Negative bf16 logits a step or two apart, fewer at a time than k."""
    g = torch.Generator(device="cuda").manual_seed(7)
    for V in (272, 494, 935, 4391, 10335, 40000):
        for spread in (0.02, 0.1, 1.0, 3.0):
            x = (offset * (1.0 + 1e-3 * spread * torch.randn((3, 1, 2, V), generator=g, device="cuda")) if abs(offset) > 100 or 0 < abs(offset) < 1
                 else offset + spread * torch.randn((3, 1, 2, V), generator=g, device="cuda")).to(dtype)
            u = torch.rand((3, 1, 2), generator=g, device="cuda")
            for k in (100, V // 2 + 1, V - 1, 1300):
                _check(gls, x, u, top_k=min(k, V - 1), top_p=0.9)
                _check(gls, x, u, top_k=min(k, V - 1))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_few_distinct_logits(gls, dtype):
    g = torch.Generator(device="cuda").manual_seed(8)
    for V in (300, 2000, 9001, 30000):
        for n, step, offset in ((1, 1.0, -5.0), (2, 0.5, -77.5), (3, 0.0625, -10.0), (17, 0.5, -90.0), (2, 1e-30, 0.0), (3, 1e-40, -1e-40)):
            x = (offset + step * torch.randint(0, n, (2, 1, 3, V), generator=g, device="cuda").float()).to(dtype)
            u = torch.rand((2, 1, 3), generator=g, device="cuda")
            for k in (40, V // 2, V - 1, min(1300, V - 1)):
                _check(gls, x, u, top_k=k)
                _check(gls, x, u, top_k=k, top_p=0.6, min_p=0.2)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_fewer_tokens_than_k(gls, dtype):
    """Rows with a few allowed tokens, the others masked."""
    g = torch.Generator(device="cuda").manual_seed(9)
    for V in (300, 4000, 30000, 128256):
        for n in (1, 3, 20, 60):
            x = torch.full((3, 1, 2, V), -math.inf, device="cuda", dtype=dtype)
            at = torch.rand((3, 1, 2, V), generator=g, device="cuda").argsort(-1)[..., :n]
            x.scatter_(-1, at, (-3.0 + torch.randn((3, 1, 2, n), generator=g, device="cuda")).to(dtype))
            u = torch.rand((3, 1, 2), generator=g, device="cuda")
            for k in (2, 17, 50, 299, 1300, 2 ** 31 - 1):
                _check(gls, x, u, top_k=k)
                _check(gls, x, u, top_k=k, top_p=0.8)
