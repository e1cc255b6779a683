"""sample_tokens at temperatures from high to hardly any, over all of the range of inv_temp, against the 64-bit form."""
import math

import pytest
import torch

from tests import vocab_ops_ref as ref

pytestmark = pytest.mark.gpu

LOW = [1e5, 1e6, 1.2e6, 1e7, 1e8, 3e8, 1e9, 1e12, 1e20]  # inverse temperatures


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _check(gls, x, u, what="", lp_more=0.0, **kw):
    got = gls.sample_tokens(x, u, **kw)
    torch.cuda.synchronize()
    if isinstance(kw.get("inv_temp"), float) and kw["inv_temp"] == ref.f32(1e-20):  # in range, as fp32 1e-20; for the 64-bit form, which takes it for less, a step more
        kw["inv_temp"] = 1.0000001e-20
    tokens, lp = ref.sample(x, u, **kw)
    assert torch.equal(got["tokens"].cpu().long(), tokens), (what, got["tokens"].cpu().flatten().tolist()[:20], tokens.flatten().tolist()[:20])
    off = (got["logprobs"].cpu().double() - lp).abs()
    assert bool((off <= ref.SLP + lp_more + ref.U * lp.abs()).all()), (what, float(off.max()))


def _rows(shape, dtype, seed):
    """Rows whose largest logits are single ones, neighbours of the type, and groups of equal ones."""
    x = 3.0 * torch.randn(shape, generator=_gen(seed), device="cuda")
    x[1] = (x[1] / 2.0).round() * 2.0
    x = x.to(dtype)
    top = x[2].amax(-1, keepdim=True)
    x[2] = torch.where(torch.rand(x[2].shape, generator=_gen(seed + 1), device="cuda") < 0.02, top, x[2])
    x[..., 3] = -math.inf
    return x


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [1000, 9001, 128256])
def test_low_temperatures(gls, V, dtype):
    for i, it in enumerate(LOW):
        x = _rows((3, 2, 2, V), dtype, 10 * V + i)
        u = torch.rand((3, 2, 2), generator=_gen(i), device="cuda")
        it = ref.f32(it)
        for kw in (dict(), dict(top_p=0.5), dict(top_p=0.9), dict(min_p=0.1), dict(top_k=7), dict(top_k=300, top_p=0.7)):
            _check(gls, x, u, (V, it, kw), inv_temp=it, **kw)
    per_row = torch.tensor(LOW[:9], device="cuda").view(9, 1, 1)
    x = _rows((9, 1, 3, V), dtype, V + 1)
    u = torch.rand((9, 1, 3), generator=_gen(99), device="cuda")
    _check(gls, x, u, (V, "per row"), inv_temp=per_row)
    _check(gls, x, u, (V, "per row"), inv_temp=per_row, top_p=torch.linspace(0.2, 1.0, 9, device="cuda"))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [1000, 9001, 300001])
def test_large_logits(gls, V, dtype):
    """Products of logit and inverse temperature around and beyond 2^24, by the logits."""
    for i, size in enumerate([1e6, 1.1e7, 1.2e7, 3e7, 1e10, 1e30]):
        x = _rows((3, 1, 2, V), torch.float32, V + i)
        x = (size * (1.0 + x * 2.0 ** -20)).to(dtype)
        x[..., V // 2:] = -x[..., V // 2:]
        x[2, ..., 5] = math.nan
        u = torch.rand((3, 1, 2), generator=_gen(i), device="cuda")
        for kw in (dict(), dict(top_p=0.5), dict(inv_temp=0.01), dict(top_p=0.9, inv_temp=3.0)):
            _check(gls, x, u, (V, size, kw), lp_more=1e-6 if V > 1 << 18 else 0.0, **kw)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_high_temperatures(gls, dtype):
    for i, it in enumerate([1e-20, 1e-10, 1e-3]):
        x = _rows((3, 1, 2, 5003), dtype, i)
        u = torch.rand((3, 1, 2), generator=_gen(i), device="cuda")
        for kw in (dict(), dict(top_k=100), dict(min_p=0.5), dict(top_k=100, top_p=0.5)):
            _check(gls, x, u, (it, kw), inv_temp=ref.f32(it), **kw)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_low_temperatures_in_a_cluster_and_beside_others(gls, dtype):
    """Rows swept by several CTAs, by one of each size, and rows of other temperatures beside them."""
    for rows in (1, 5, 74, 200, 700):
        x = _rows((3, rows, 1, 9001), dtype, rows)[2].unsqueeze(0).transpose(0, 1)
        it = torch.tensor([1.0, 3e8, math.inf, 1e12, 0.5], device="cuda").repeat(140)[:rows]
        u = torch.rand((rows, 1, 1), generator=_gen(rows), device="cuda")
        _check(gls, x, u, rows, inv_temp=it)
        _check(gls, x, u, rows, inv_temp=it, top_p=0.3)
