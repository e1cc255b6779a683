"""sample_tokens against a 64-bit form of its definition: tokens equal, log probabilities within the tolerance
derived in vocab_ops_ref.py."""
import pytest
import torch

from tests import vocab_ops_ref as ref

pytestmark = pytest.mark.gpu

INF = float("inf")
SETTINGS = [dict(), dict(top_k=1), dict(top_k=5), dict(top_k=50), dict(top_p=0.9), dict(top_p=0.999), dict(min_p=0.05),
            dict(top_k=40, top_p=0.8), dict(top_k=700, top_p=0.95, min_p=0.01), dict(top_p=0.7, min_p=0.3),
            dict(top_k=3, min_p=0.5), dict(inv_temp=INF), dict(top_p=1e-6), dict(min_p=1.0)]


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _logits(shape, dtype, seed, spread=3.0, step=None):
    x = spread * torch.randn(shape, generator=_gen(seed), device="cuda")
    if step:  # many equal logits
        x = (x / step).round() * step
    return x.to(dtype)


def _check(gls, x, u, what="", lp_more=0.0, **kw):
    got = gls.sample_tokens(x, u, **kw)
    torch.cuda.synchronize()
    tokens, lp = ref.sample(x, u, **kw)
    assert torch.equal(got["tokens"].cpu().long(), tokens), (what, got["tokens"].cpu().flatten().tolist()[:20], tokens.flatten().tolist()[:20])
    off = (got["logprobs"].cpu().double() - lp).abs()
    tol = ref.SLP + lp_more + ref.U * lp.abs()
    assert bool((off <= tol).all()), (what, float(off.max()))
    return got


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [1, 2, 7, 255, 256, 257, 1000, 8192, 8193, 50257])
def test_sizes(gls, V, dtype):
    for i, kw in enumerate(SETTINGS):
        x = _logits((3, 2, 2, V), dtype, 100 * V + i, spread=[1.0, 3.0, 6.0][i % 3])
        u = torch.rand((3, 2, 2), generator=_gen(i), device="cuda")
        kw = dict(dict(inv_temp=[1.0, 0.7, 1.6][i % 3]), **kw)
        _check(gls, x, u, "%d %s" % (V, kw), **kw)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [5, 300, 9001])
def test_equal_logits(gls, V, dtype):
    """Rows of few distinct values, of one value, and with zeros of both signs: ties stay by the lowest index."""
    for i, kw in enumerate(SETTINGS + [dict(top_k=V // 2), dict(top_k=V - 1, top_p=0.5), dict(top_p=0.5)]):
        x = _logits((4, 1, 2, V), dtype, V + i, step=2.0)
        x[1] = 0.25
        x[2, :, :, ::3] = -0.0
        u = torch.rand((4, 1, 2), generator=_gen(i), device="cuda")
        u[1, 0, 0], u[1, 0, 1] = 0.5, 0.0
        _check(gls, x, u, "%d %s" % (V, kw), **kw)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_long_rows(gls, dtype):
    for V in (152064, 300001):
        for i, kw in enumerate([dict(), dict(top_k=50, top_p=0.9), dict(top_p=0.95), dict(top_k=2000), dict(min_p=0.02),
                                dict(top_k=100000, top_p=0.99)]):
            x = _logits((1, 2, 1, V), dtype, V + i)
            x[0, 1, 0] *= 0.1  # a flat row
            u = torch.rand((1, 2, 1), generator=_gen(i), device="cuda")
            _check(gls, x, u, "%d %s" % (V, kw), lp_more=1e-6, **kw)


def test_chunks_of_many_tokens(gls):
    V = (1 << 21) + 13  # more than 1024 chunks of 1024
    x = _logits((1, 1, 3, V), torch.bfloat16, 5)
    u = torch.tensor([[[0.1, 0.6, 0.99]]], device="cuda")
    for kw in (dict(), dict(top_k=300), dict(top_p=0.9), dict(min_p=0.1)):
        _check(gls, x, u, str(kw), lp_more=1e-5, **kw)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_masked_logits(gls, dtype):
    x = _logits((6, 1, 1, 3001), dtype, 7)
    x[0, ..., 100:] = -INF
    x[1] = -INF                      # nothing left
    x[2] = -INF
    x[2, ..., 2999] = -3.0           # one token
    x[3, ..., ::2] = float("nan")
    x[3, ..., 1::4] = INF
    x[4] = torch.finfo(dtype).min    # the type's lowest value is a logit like others
    x[4, ..., 17] = -INF
    x[5, ..., 5] = torch.finfo(dtype).max
    u = torch.full((6, 1, 1), 0.75, device="cuda")
    for kw in SETTINGS:
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        got = gls.sample_tokens(x, u, status=status, **kw)
        tokens, lp = ref.sample(x, u, **kw)
        assert torch.equal(got["tokens"].cpu().long(), tokens), kw
        assert bool(((got["logprobs"].cpu().double() - lp).abs() <= ref.SLP + ref.U * lp.abs()).all()), kw
        assert int(status) == gls.DEV_EMPTY_SUPPORT


def test_ends_of_the_unit_interval(gls):
    x = _logits((2, 1, 4, 5000), torch.bfloat16, 9)
    x[..., :3] = -INF
    x[..., -2:] = -INF
    u = torch.tensor([0.0, 1.0 - 2.0 ** -24, 1.0, 0.5], device="cuda").expand(2, 1, 4).contiguous()
    for kw in SETTINGS:
        _check(gls, x, u, str(kw), **kw)


def test_settings_per_row(gls):
    B, K, J, V = 6, 3, 2, 4000
    x = _logits((B, K, J, V), torch.bfloat16, 11)
    g = _gen(12)
    u = torch.rand((B, K, J), generator=g, device="cuda")
    it = torch.tensor([1.0, 0.5, INF, 2.0, 1.0, 0.8], device="cuda")
    k = torch.randint(0, 100, (B, K), generator=g, device="cuda", dtype=torch.int32)
    p = 0.2 + 0.9 * torch.rand((B, K, J), generator=g, device="cuda")
    m = torch.tensor([[[0.0, 0.1]]], device="cuda")
    _check(gls, x, u, inv_temp=it, top_k=k, top_p=p, min_p=m)
    _check(gls, x, u, inv_temp=it.repeat(2)[::2], top_k=k.T.contiguous().T, top_p=p.transpose(0, 2).contiguous().transpose(0, 2))


def test_settings_out_of_range(gls):
    x = _logits((8, 1, 1, 600), torch.float32, 13)
    u = torch.full((8, 1, 1), 0.3, device="cuda")
    nan = float("nan")
    cases = dict(inv_temp=[1.0, 0.0, -1.0, nan, 1e-30, 1e30, -INF, 2.0], top_p=[1.0, 0.0, -0.5, nan, 2.0, 1.0, 1.0, 0.5],
                 min_p=[0.0, -0.1, 1.5, nan, 0.1, 1.0, 0.0, 0.0])
    for name, v in cases.items():
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        kw = {name: torch.tensor(v, device="cuda")}
        got = gls.sample_tokens(x, u, status=status, **kw)
        tokens, _ = ref.sample(x, u, **kw)
        assert torch.equal(got["tokens"].cpu().long(), tokens), name
        assert int(status) == gls.DEV_BAD_SETTING
        assert bool((got["logprobs"].cpu()[tokens < 0] == 0).all())
    bad = torch.tensor([0.5, -0.1, 1.1, nan, INF, 0.0, 1.0, 0.2], device="cuda").view(8, 1, 1)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = gls.sample_tokens(x, bad, status=status)
    assert (got["tokens"].view(-1) < 0).tolist() == [False, True, True, True, True, False, False, False]
    assert int(status) == gls.DEV_BAD_SETTING


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_strides_and_alignment(gls, dtype):
    store = _logits((2, 5, 3, 1203), dtype, 15)
    u = torch.rand((2, 5, 3), generator=_gen(16), device="cuda")
    for off in range(0, 9):
        _check(gls, store[..., off:off + 1190], u, "offset %d" % off, top_k=30, top_p=0.9)
    _check(gls, store.transpose(0, 1)[:, :, ::2], u.transpose(0, 1)[:, :, ::2].contiguous(), min_p=0.02)
    one = store[:, :1].expand(2, 5, 3, 1203)  # every draft draws from one row
    _check(gls, one, u, top_p=0.95)


def test_what_is_around_the_rows_is_not_read(gls):
    """Positions in front of and behind a row hold +largest values: none may win."""
    store = torch.full((4, 1, 1, 1000), 3e38, device="cuda")
    for lo, n in ((1, 998), (3, 513), (5, 17), (2, 1)):
        x = store[..., lo:lo + n]
        x.copy_(_logits((4, 1, 1, n), torch.float32, n))
        _check(gls, x, torch.full((4, 1, 1), 0.9, device="cuda"), top_p=0.9)
        x.fill_(3e38)


def test_outputs_given_streams_and_graphs(gls):
    x = _logits((4, 2, 1, 20000), torch.bfloat16, 17)
    u = torch.rand((4, 2, 1), generator=_gen(18), device="cuda")
    kw = dict(top_k=200, top_p=0.9, inv_temp=torch.tensor([1.0, 2.0, INF, 0.5], device="cuda"))
    want = gls.sample_tokens(x, u, **kw)
    out = dict(tokens=torch.full((4, 2, 1), -7, dtype=torch.int32, device="cuda"))
    assert gls.sample_tokens(x, u, out=out, **kw) is out
    assert torch.equal(out["tokens"], want["tokens"])
    assert "logprobs" not in gls.sample_tokens(x, u, want_logprobs=False)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = gls.sample_tokens(x, u, **kw)
    side.synchronize()
    assert torch.equal(got["tokens"], want["tokens"]) and torch.equal(got["logprobs"], want["logprobs"])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = gls.sample_tokens(x, u, **kw)
    x2, u2 = _logits((4, 2, 1, 20000), torch.bfloat16, 19), torch.rand((4, 2, 1), generator=_gen(20), device="cuda")
    x.copy_(x2)
    u.copy_(u2)
    graph.replay()
    torch.cuda.synchronize()
    tokens, _ = ref.sample(x2, u2, **kw)
    assert torch.equal(held["tokens"].cpu().long(), tokens)
    for _ in range(3):
        again = gls.sample_tokens(x, u, **kw)
        assert torch.equal(again["tokens"], held["tokens"]) and torch.equal(again["logprobs"], held["logprobs"])


def test_frequencies(gls):
    """The kept tokens come as often as their weights say: 20000 draws, each count within 6 standard deviations."""
    row = torch.tensor([0.0, 1.0, 2.0, -1.0, 1.5, -INF, 0.5], device="cuda")
    n = 20000
    x = row.view(1, 1, 1, 7).expand(1, 1, n, 7)
    u = torch.rand((1, 1, n), generator=_gen(21), device="cuda")
    got = gls.sample_tokens(x, u, top_k=4)["tokens"].flatten().long().cpu()
    w = torch.exp(row.double().cpu())
    w[[0, 3]] = 0
    p = w / w.sum()
    count = torch.bincount(got, minlength=7).double()
    assert bool(((count - n * p).abs() <= 6 * (n * p * (1 - p)).sqrt()).all())


def test_refusals(gls):
    x, u = torch.zeros((1, 1, 1, 8), device="cuda"), torch.zeros((1, 1, 1), device="cuda")
    bad = [dict(uniforms=u[0]), dict(uniforms=u.double()), dict(uniforms=u.cpu()), dict(logits=x.half()), dict(logits=x[0]),
           dict(inv_temp=0.0), dict(inv_temp=float("nan")), dict(inv_temp=1e30), dict(top_p=0.0), dict(min_p=-1.0), dict(min_p=2.0),
           dict(top_k=torch.zeros(1, device="cuda")), dict(top_p=torch.ones(2, device="cuda")),
           dict(inv_temp=torch.ones(1)), dict(min_p=torch.zeros((1, 1, 1, 1), device="cuda")),
           dict(status=torch.zeros(2, dtype=torch.int32, device="cuda")), dict(out=dict(tokens=torch.zeros(1, device="cuda"))),
           dict(logits=x.clone().requires_grad_())]
    for kw in bad:
        a = dict(logits=x, uniforms=u)
        a.update(kw)
        with pytest.raises(gls.GlsError):
            gls.sample_tokens(**a)
    with torch.no_grad():
        gls.sample_tokens(x.clone().requires_grad_(), u)


@pytest.mark.parametrize("most,inv_temp,min_p", [(3.3137195, 0.10763583, 0.7), (3.4443467, 0.103553735, 0.7), (2.37963, 0.9676231, 0.1),
                                                 (2.776235, 0.82939124, 0.1)])
def test_border_of_min_p_around_zero(gls, most, inv_temp, min_p):
    """ln(min_p) / inv_temp + the largest logit is zero but for 1e-15: the 64-bit difference holds up to a million
    neighbouring codes for equal.  Logits around it, and far smaller than that difference's step."""
    x = torch.tensor([most, 0.0, 1e-30, -1e-30, 1e-14, -1e-14, 1e-8, -1e-8, -2.4424904e-15, 1e-45, -1.0, most / 2] * 3, device="cuda")
    x = x.view(1, 1, 1, 36).expand(1, 1, 64, 36).contiguous()
    u = ((torch.arange(64, device="cuda") + 0.5) / 64).view(1, 1, 64)
    _check(gls, x, u, inv_temp=ref.f32(inv_temp), min_p=ref.f32(min_p))


def test_top_k_beyond_32_bits(gls):
    x, u = _logits((2, 1, 8, 500), torch.float32, 31), torch.rand((2, 1, 8), generator=_gen(32), device="cuda")
    want = gls.sample_tokens(x, u)
    for k in (2 ** 31, 2 ** 40 + 5, -2 ** 40 + 5):
        assert torch.equal(gls.sample_tokens(x, u, top_k=k)["tokens"], want["tokens"])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_more_rows_than_multiprocessors(gls, dtype):
    """Rows of more than 8192 tokens by each size of CTA: between one and four a multiprocessor the settings choose."""
    for rows in (200, 700):
        x, u = _logits((rows, 1, 1, 9001), dtype, 41), torch.rand((rows, 1, 1), generator=_gen(42), device="cuda")
        for kw in (dict(), dict(top_k=50, top_p=0.9), dict(min_p=0.05), dict(top_p=0.9), dict(top_p=0.9, min_p=0.05), dict(inv_temp=INF),
                   dict(top_k=torch.full((rows,), 50, dtype=torch.int32, device="cuda"))):
            _check(gls, x, u, what=(rows, kw.keys()), **kw)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [1909, 37903])
def test_a_token_kept_alone_has_log_probability_zero(gls, V, dtype):
    x, u = _logits((24, 2, 1, V), dtype, 51, spread=4.0), torch.rand((24, 2, 1), generator=_gen(52), device="cuda")
    per_row = torch.ones(24, dtype=torch.int32, device="cuda")
    for kw in (dict(top_k=1), dict(top_k=1, top_p=0.9, min_p=0.02, inv_temp=2.0), dict(inv_temp=INF), dict(top_k=per_row, inv_temp=0.8),
               dict(top_p=1e-6, inv_temp=1.25)):
        lp = gls.sample_tokens(x, u, **kw)["logprobs"]
        assert torch.equal(lp, torch.zeros_like(lp)), (kw.keys(), float(lp.min()), float(lp.max()))
    for kw in (dict(), dict(top_k=50), dict(top_p=0.9), dict(inv_temp=20.0), dict(min_p=0.05, inv_temp=20.0)):
        assert bool((gls.sample_tokens(x, u, **kw)["logprobs"] <= 0).all()), kw
