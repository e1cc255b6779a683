"""sample_tokens at the ends of the unit interval: the first and the last kept token by index, however little weight they have."""
import math

import pytest
import torch

from tests import vocab_ops_ref as ref

pytestmark = pytest.mark.gpu


def _ends(x, u, it, top_k=0, top_p=1.0, min_p=0.0):
    """(token, log probability) of a row for u = 0 or 1 from its kept tokens themselves (partial sums of a parallel scan may pass
    their total, so that one in front of the last seems to exceed it)."""
    x = x.double()
    order = x.sort(descending=True, stable=True).indices[: int(torch.isfinite(x).sum())]
    z = (x[order] - x[order[0]]) * it
    w = torch.exp(z)
    n = min(len(order), top_k) if 0 < top_k < x.numel() else len(order)
    if top_p < 1:
        cum = torch.cumsum(w[:n].cpu(), 0)
        n = max(1, int((cum - w[:n].cpu() < ref.f32(top_p) * cum[-1]).sum()))
    if min_p > 0:
        n = max(1, min(n, int((z >= math.log(ref.f32(min_p))).sum())))
    at = order[:n][w[:n] > 0]
    t = int(at.min() if u == 0 else at.max())
    return t, float((x[t] - x[order[0]]) * it - torch.log(w[:n].sum()))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [2, 7, 300, 5000, 9001, 50257, 300001])
def test_first_and_last(gls, V, dtype):
    """Weights down to 2^-750 of the largest, beside sums that would round them away."""
    g = torch.Generator(device="cuda").manual_seed(V)
    for rows in (2, 100):
        if rows * V > 3e6:
            continue
        x = (3.0 * torch.randn((rows, 1, 4, V), generator=g, device="cuda")).clamp(-12, 12).to(dtype)
        x[0, 0, 0, V // 2:] = -math.inf
        x[1, 0, 3, :V // 2] = -math.inf
        x[1, 0, 0] = x[1, 0, 0, 0]  # all equal
        u = torch.tensor([0.0, 1.0, 0.0, 1.0], device="cuda").expand(rows, 1, 4).contiguous()
        for it in (1.0, 4.0, 20.0):
            for kw in (dict(), dict(top_k=3), dict(top_k=200), dict(top_k=3000), dict(top_k=40, top_p=0.9), dict(top_p=0.99), dict(min_p=1e-30),
                       dict(top_p=0.9999999), dict(top_k=V - 1)):
                got = gls.sample_tokens(x, u, inv_temp=it, **kw)
                n = 2  # rows compared
                want = [_ends(row, end, it, **kw) for row, end in zip(x[:n].reshape(4 * n, V), u[:n].flatten().tolist())]
                tokens, lp = torch.tensor([t for t, _ in want]).view(n, 1, 4), torch.tensor([y for _, y in want], dtype=torch.float64).view(n, 1, 4)
                assert torch.equal(got["tokens"][:n].cpu().long(), tokens), (rows, it, kw, got["tokens"][:n].flatten().tolist(), tokens.flatten().tolist())
                off = (got["logprobs"][:n].cpu().double() - lp).abs()
                assert bool((off <= ref.SLP + 1e-6 + ref.U * lp.abs()).all()), (it, kw)


def test_weights_that_64_bits_do_not_hold(gls):
    """Tokens below 2^-1000 of the first are no tokens to draw."""
    x = torch.full((1, 1, 2, 5000), -2000.0, device="cuda")
    x[..., 700], x[..., 900], x[..., 4000] = 0.0, -600.0, -690.0
    u = torch.tensor([[[0.0, 1.0]]], device="cuda")
    for kw in (dict(), dict(top_k=30), dict(top_k=4000), dict(min_p=0.0)):
        got = gls.sample_tokens(x, u, **kw)
        assert got["tokens"].flatten().tolist() == [700, 4000], kw
        assert torch.allclose(got["logprobs"].cpu().flatten(), torch.tensor([0.0, -690.0]))
