"""The sums behind sample_tokens: borders of top-p and draws next to borders, where a row's total has to be good to what the
kernel takes it to be, and log probabilities of plain draws, whose total is the sweep's.

Tolerance of those log probabilities (fixed before the first run), u = 2^-24: a set of 1024 tokens is a sum of exponentials
that are off by 1.5e-7 (measured for every fp32 argument), whose exponents t have two roundings, (a c2 - ref) and c2's own, u |t|
each, where |t| is 6.4 at most on the mean weighted by the terms (one term 1 and 1023 of 2^-7.85), 0.5 more for the reference's
rounding; ten additions: 1.5e-7 + u (10 + 13.3 ln 2) = 1.3e-6 = SET.  Sets of more tokens have three roundings of exponents, a mean that grows by 1 for
each doubling, and fewer additions: 2.1 u more for each.  The own set of a token with more than half of the total is summed in 64 bits,
so that the total is off by SET times what others hold, at most 1 - p of it; then half a step of the result."""
import math

import pytest
import torch

from tests import vocab_ops_ref as ref

pytestmark = pytest.mark.gpu

SET = 1.5e-7 + ref.U * (10.0 + 13.3 * math.log(2.0))


def _weights(row, it):
    x = row.double()
    return torch.exp((x - x.max()) * it)


def _peaked(V, below, at=77):
    row = torch.full((V,), 0.25 - below, device="cuda")
    row[at] = 0.25
    return row


# the first four times log2(e) are 5.9e-8 off as fp32, either way
ROUNDED = [0.6963212, 0.6951287, 0.6941785, 1.3899848, 0.75, 0.9, 1.0]


@pytest.mark.parametrize("below", [12.0, 14.5, 16.0])
@pytest.mark.parametrize("inv_temp", ROUNDED)
def test_border_of_top_p_in_a_flat_row(gls, inv_temp, below):
    """One token `below` exponents above 152063 equal ones and 8192 shares: u = 1 draws the last token that stays."""
    it, n = ref.f32(inv_temp), 8192
    for dtype in (torch.float32, torch.bfloat16):
        row = _peaked(152064, below * math.log(2.0) / it).to(dtype)
        w = _weights(row, it)
        p = torch.linspace(0.45, 0.9999, n, dtype=torch.float32, device="cuda")
        x = row.view(1, 1, 1, -1).expand(n, 1, 1, -1)
        got = gls.sample_tokens(x, torch.ones((n, 1, 1), device="cuda"), inv_temp=it, top_p=p)["tokens"].flatten().long()
        order = row.double().sort(descending=True, stable=True).indices
        cum = torch.cumsum(w[order], 0)
        kept = torch.searchsorted(cum, p.double() * cum[-1]) + 1  # tokens whose mass in front is below the goal
        want = torch.cummax(order, 0).values[kept.clamp(max=len(order)) - 1]
        assert torch.equal(got, want), (dtype, int((got != want).sum()), float((got - want).abs().max()))


@pytest.mark.parametrize("below", [1.0, 14.5, 20.0])
@pytest.mark.parametrize("inv_temp", [0.6963212, 0.6951287, 1.0])
def test_draws_from_a_flat_row(gls, inv_temp, below):
    it, n = ref.f32(inv_temp), 20000
    for V, dtype in ((152064, torch.float32), (152064, torch.bfloat16), (50257, torch.float32)):
        row = _peaked(V, below * math.log(2.0) / it, at=V // 3).to(dtype)
        g = torch.Generator(device="cuda").manual_seed(V)
        u = torch.rand((1, 1, n), generator=g, device="cuda")
        u[..., :3] = torch.tensor([0.0, 1.0, 1.0 - 2.0 ** -24], device="cuda")
        got = gls.sample_tokens(row.view(1, 1, 1, -1).expand(1, 1, n, -1), u, inv_temp=it)
        cum = torch.cumsum(_weights(row, it), 0)
        want = torch.searchsorted(cum, u.flatten().double() * cum[-1], right=True).clamp(max=V - 1)
        assert torch.equal(got["tokens"].flatten().long(), want), int((got["tokens"].flatten().long() != want).sum())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [700, 32000, 152064, 300001])
def test_log_probabilities_of_plain_draws(gls, V, dtype):
    """Rows of normal logits of several deviations, flat ones with a peak, and rows in which one token has nearly all, at
    inverse temperatures from 0.5 to 2 in small steps."""
    steps = 61
    g = torch.Generator(device="cuda").manual_seed(V)
    z = torch.randn(V, generator=g, device="cuda")
    more = 2.1 * ref.U * max(0, math.ceil(math.log2((V + 7) / (256 * 1024))))
    for name, row in (("1", z), ("3", 3 * z), ("6", 6 * z), ("flat", _peaked(V, 11.0)), ("peak", z + _peaked(V, 30.0)), ("two", 0.1 * z + _peaked(V, 14.0))):
        row = row.to(dtype)
        it = torch.linspace(0.5, 2.0, steps, device="cuda")
        u = torch.rand((steps, 1, 8), generator=g, device="cuda")
        got = gls.sample_tokens(row.view(1, 1, 1, -1).expand(steps, 1, 8, -1), u, inv_temp=it)
        worst = 0.0
        for i in range(steps):
            x = row.double()
            d = (x - x.max()) * float(it[i])
            lse = torch.log1p(torch.exp(d).sum() - 1.0)
            t = got["tokens"][i, 0].long()
            lp = d[t] - lse
            p = torch.exp(lp)
            tol = (SET + more) * torch.where(p > 0.5, 1.0 - p, torch.ones_like(p)) * (1.0 + 1e-3) + ref.U * lp.abs() + 1e-12
            off = (got["logprobs"][i, 0].double() - lp).abs()
            worst = max(worst, float((off / tol).max()))
        assert worst <= 1.0, (name, worst)
