"""The embedding gradient on whole numbers.  Every sum of these is exact in fp32 (below 2^24 with any of its
partial sums), and so is its product with a power of two, so the result has to be equal: a position left out,
taken twice or given to another token shows, however often a token occurs."""
import pytest
import torch

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _check(gls, tok, V, D, dtype, out_dtype, seed, pad=0):
    N = tok.numel()
    assert 8 * N * 2 < 1 << 24
    n = torch.randint(-8, 9, (N, D), generator=_gen(seed), device="cuda")
    g = torch.full((N, D + pad), float("nan"), dtype=dtype, device="cuda")[:, :D]
    g.copy_(n)
    live = (tok >= 0) & (tok < V)
    want = torch.zeros((V, D), dtype=torch.int64, device="cuda").index_add_(0, tok.long()[live], n[live])
    half = (want.double() * 0.5).to(out_dtype)  # exact in fp32; to bf16 one rounding of the exact value
    out = torch.full((V, D + pad), 3.0, dtype=out_dtype, device="cuda")[:, :D]
    gls.embed_tokens_backward(g, tok, V, scale=0.5, grad_table=out)
    assert torch.equal(out, half), (N, V, D, int((out != half).any(1).sum()))
    if out_dtype is F:  # on top of what is there
        gls.embed_tokens_backward(g, tok, V, scale=-2.0, grad_table=out, accumulate=True)
        assert torch.equal(out, (want.double() * -1.5).to(F))


def _zipf(N, V, seed, none=0.05):
    r = torch.exp(torch.rand(N, generator=_gen(seed), device="cuda", dtype=torch.float64) * torch.log(torch.tensor(float(V + 1))))
    t = (r.long().clamp(1, V) - 1) * 7919 % V
    return torch.where(torch.rand(N, generator=_gen(seed + 1), device="cuda") < none, torch.full_like(t, -1), t).to(torch.int32)


@pytest.mark.parametrize("dtype,out_dtype", [(F, F), (BF, BF), (BF, F)])
@pytest.mark.parametrize("N,V,D,pad", [
    (400000, 200, 8, 0),         # one pass over the digits; the commonest token goes on over 700 ranges and more
    (150000, 5000, 16, 0), (140001, 3, 33, 0), (131072, 900, 8, 3), (131073, 900, 8, 0),
    (16384, 700, 40, 0), (16385, 700, 40, 0), (20000, 70000, 7, 1), (200000, 3000000, 8, 0),
    (1000000, 17, 8, 0), (20000, (1 << 27) + 5, 1, 0),   # four passes
])
def test_whole_numbers(gls, dtype, out_dtype, N, V, D, pad):
    _check(gls, _zipf(N, V, N), V, D, dtype, out_dtype, 5, pad)


@pytest.mark.parametrize("D", [16, 21, 1030])
@pytest.mark.parametrize("dtype", [F, BF])
def test_tokens_over_a_few_and_many_ranges(gls, dtype, D):
    """Runs that end at, before and behind the ends of the ranges (8 positions here), over as many of them as
    are joined by a thread and by the warps of a CTA."""
    runs = [1, 7, 8, 9, 15, 16, 17, 8 * 31, 8 * 32, 8 * 33, 8 * 33 + 1, 8 * 34 - 1, 8 * 34, 3, 8 * 65 + 2, 5, 2048, 1, 2, 4099, 6]
    tok = torch.cat([torch.full((n,), 3 * i, dtype=torch.int32) for i, n in enumerate(runs)])
    for seed, lead in ((0, 0), (1, 3)):  # and the same from another place in the first range
        t = torch.cat([torch.zeros(lead, dtype=torch.int32), tok])
        t = t[torch.randperm(t.numel(), generator=torch.Generator().manual_seed(seed))].cuda()
        _check(gls, t, 3 * len(runs), D, dtype, F, seed)
    many = torch.full((30000,), 4, dtype=torch.int32, device="cuda")  # a single token, through the larger sort
    _check(gls, many, 6, D, dtype, F, 9)
