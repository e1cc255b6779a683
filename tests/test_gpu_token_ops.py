"""Log probabilities of tokens, the embedding lookup and their gradients against plain 64-bit forms
(tests/token_ops_ref.py, where the tolerances are derived)."""
import pytest
import torch

from tests import token_ops_ref as ref

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32
INF = float("inf")


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _logits(shape, dtype, seed, sd=4.0):
    x = sd * torch.randn(shape, generator=_gen(seed), device="cuda")
    x += 8.0 * (torch.rand(shape, generator=_gen(seed + 1), device="cuda") < 0.01)
    return x.to(dtype)


def _tokens(shape, V, seed, none=0.1):
    t = torch.randint(V, shape, generator=_gen(seed), device="cuda")
    return torch.where(torch.rand(shape, generator=_gen(seed + 1), device="cuda") < none,
                       torch.full_like(t, -1), t).to(torch.int32)


def _inv(B, K, J, inv_temp=1.0, per=None):
    v = torch.full((K,), ref.f32(inv_temp), dtype=torch.float64) if per is None else torch.tensor(
        [ref.f32(x) for x in per], dtype=torch.float64)
    return v[None, :, None].expand(B, K, J).contiguous().cuda()


def _check(gls, x, tok, M, inv_temp=1.0, per=None, what=""):
    B, K, J, V = x.shape
    got = gls.token_logprobs(x, tok, top=M, inv_temp=inv_temp, inv_temp_per_draft=per)
    t = tok if tok.dim() == 4 else tok[..., None]
    want = ref.logprobs(x, t, _inv(B, K, J, inv_temp, per), M)
    want["logprobs"] = want["logprobs"].view(got["logprobs"].shape)
    ref.check_logprobs(got, want, what)
    return got


# ---- log probabilities --------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [F, BF])
@pytest.mark.parametrize("V", [1, 2, 15, 16, 17, 33, 511, 513, 1024, 2047, 2049, 4099, 30011])
def test_logprobs_sizes(gls, dtype, V):
    for n, (B, K, J, M) in enumerate([(1, 1, 1, 0), (2, 3, 2, 5), (1, 2, 3, 1)]):
        x = _logits((B, K, J, V), dtype, 10 * V + n)
        _check(gls, x, _tokens((B, K, J), V, V + n), M, 1.25, what="V=%d M=%d %s" % (V, M, dtype))


@pytest.mark.parametrize("dtype", [F, BF])
@pytest.mark.parametrize("V", [300, 513, 700, 1000, 1025, 1817, 2049, 4500, 9000, 17000])
def test_logprobs_many_alternatives_of_short_rows(gls, dtype, V):
    for M in (24, 25, 50, 129, 256):
        x = _logits((5, 2, 3, V + 5), dtype, V + M)[..., 2:V + 2]
        x[0, 0, 0, :V - M // 2] = -INF       # fewer alternatives than asked for
        x[0, 0, 1] = 0.25                    # all equal: the lowest indices
        x[0, 0, 2, ::7] = float("-inf")
        x[0, 1, 0, 3::5] = float("nan")    
        x[0, 1, 1, 5] = INF
        x[0, 1, 2] = x[0, 1, 2].round()      # many equal values
        x = x.clone() if M == 25 else x
        got = gls.token_logprobs(x, _tokens((5, 2, 3), V, M), top=M, inv_temp=1.25)
        live = x.float().masked_fill(~torch.isfinite(x), -INF).view(-1, V)
        order = torch.sort(live, dim=-1, descending=True, stable=True)
        n = min(M, V)
        ids = torch.where(order.values[:, :n] > -INF, order.indices[:, :n], -1)
        assert torch.equal(got["top_ids"].view(-1, M)[:, :n].long(), ids), (V, M)
        assert (got["top_ids"].view(-1, M)[:, n:] == -1).all()
        rest = x[1:].contiguous()
        _check(gls, rest, _tokens((4, 2, 3), V, M), M, 1.25, what="V=%d M=%d %s" % (V, M, dtype))


@pytest.mark.parametrize("dtype", [F, BF])
@pytest.mark.parametrize("V", [6150, 10189, 12420, 16385, 33000, 61898])
def test_logprobs_short_last_step(gls, dtype, V):
    for B, M in [(1, 33), (7, 50), (90, 50), (3, 256)]:
        x = _logits((B, 1, 1, V), dtype, V + M)
        x[0, 0, 0, -100:] += 20  # the last step has the best
        _check(gls, x, _tokens((B, 1, 1), V, M), M, 1.25, what="V=%d M=%d %s" % (V, M, dtype))


@pytest.mark.parametrize("dtype", [F, BF])
@pytest.mark.parametrize("M", [20, 64, 65, 128, 129, 256])
def test_logprobs_alternatives(gls, dtype, M):
    for B, K, J, V in [(1, 1, 1, 152064), (1, 2, 1, 200), (3, 1, 2, 20000)]:
        x = _logits((B, K, J, V), dtype, M)
        _check(gls, x, _tokens((B, K, J), V, M), M, what="M=%d V=%d %s" % (M, V, dtype))


@pytest.mark.parametrize("dtype", [F, BF])
def test_logprobs_many_rows(gls, dtype):
    """Enough rows that none is cut into slices, and so many that warps take several each."""
    for B, K, J, V, M in [(300, 4, 2, 3001, 5), (700, 2, 4, 1200, 20), (330, 4, 2, 6000, 0)]:
        x = _logits((B, K, J, V), dtype, V)
        _check(gls, x, _tokens((B, K, J), V, 3), M, 0.7, what="rows V=%d %s" % (V, dtype))


@pytest.mark.parametrize("dtype", [F, BF])
def test_logprobs_several_tokens_and_temperatures(gls, dtype):
    B, K, J, V = 2, 3, 2, 5003
    x = _logits((B, K, J, V), dtype, 5)
    for G in (1, 2, 33, 64):
        tok = _tokens((B, K, J, G), V, G)
        tok[0, 0, 0] = 17  # the same token again and again
        _check(gls, x, tok, 3, per=[0.5, 1.0, 2.0], what="G=%d" % G)
    none = gls.token_logprobs(x, None, top=2, want_entropy=False)
    assert none["logprobs"].shape == (B, K, J, 0) and "entropy" not in none
    want = ref.logprobs(x, torch.zeros((B, K, J, 1), device="cuda"), _inv(B, K, J), 2)
    ref.near(none["lse"], want["lse"], ref.LSE + ref.U * want["lse"].abs(), "lse without entropy")
    assert torch.equal(none["top_ids"].long(), want["top_ids"])


@pytest.mark.parametrize("dtype", [F, BF])
def test_logprobs_strides(gls, dtype):
    """Rows that start anywhere, swapped and broadcast dimensions."""
    base = _logits((2, 3, 4, 3000 + 40), dtype, 6)
    for off in (1, 3, 8, 15, 17):
        x = base[..., off:off + 3000]
        _check(gls, x, _tokens((2, 3, 4), 3000, off), 20, what="offset %d" % off)
    x = base.permute(2, 1, 0, 3)
    _check(gls, x, _tokens((4, 3, 2), 3040, 1), 5, what="permuted")
    x = base[:, :1].expand(2, 5, 4, 3040)
    _check(gls, x, _tokens((2, 5, 4), 3040, 2), 5, what="shared by the drafts")
    x = base[:1, :1, :1, :].expand(3, 2, 2, 3040)
    _check(gls, x, _tokens((3, 2, 2), 3040, 2), 5, what="one row")
    x = base[:, ::2, 1::2]
    _check(gls, x, _tokens((2, 2, 2), 3040, 2), 5, what="every second")


def _special(dtype, V):
    """Rows with masks, infinities, NaN, lowest values, ties, huge and offset logits."""
    low, high = torch.finfo(dtype).min, torch.finfo(dtype).max
    r = _logits((16, V), F, 77)
    r[0] = -INF
    r[1] = -INF
    r[1, V // 2] = 3.0
    r[2, ::2] = float("nan")
    r[2, 1] = INF
    r[3] = float("nan")
    r[4] = INF
    r[5] = low
    r[6] = low
    r[6, V - 1] = 0.0
    r[7] = 0.0
    r[7, ::3] = -0.0
    r[8] += 1.0e4
    r[9] = high
    r[10, : V - 3] = -INF
    r[11] = torch.arange(V, device="cuda") * 0.01
    r[12] = -torch.arange(V, device="cuda") * 0.01
    r[13] = -INF
    r[13, 0], r[13, V - 1] = low, low
    r[14] = low
    r[14, 5 % V] = high
    r[15] = (torch.arange(V, device="cuda") % 7).float()
    return r.to(dtype)


@pytest.mark.parametrize("dtype", [F, BF])
@pytest.mark.parametrize("V", [40, 2100, 20011])
def test_logprobs_special_rows(gls, dtype, V):
    x = _special(dtype, V).view(2, 2, 4, V)
    tok = _tokens((2, 2, 4, 3), V, 1)
    tok[..., 0] = V // 2
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    for M in (0, 20, 50):
        got = gls.token_logprobs(x, tok, top=M, status=status)
        ref.check_logprobs(got, ref.logprobs(x, tok, _inv(2, 2, 4), M), "special V=%d M=%d %s" % (V, M, dtype))
        plain = gls.token_logprobs(x, tok, top=M, want_entropy=False)
        assert torch.equal(plain["lse"], got["lse"]) or bool(
            ((plain["lse"] == got["lse"]) | ((plain["lse"] - got["lse"]).abs() <= 2e-5 + 2e-7 * got["lse"].abs())).all())
    assert int(status.item()) == gls.DEV_EMPTY_SUPPORT
    # the same rows many times over: no slices
    many = x.reshape(1, 1, 16, V).expand(200, 1, 16, V)
    t2 = tok.reshape(1, 1, 16, 3).expand(200, 1, 16, 3).contiguous()
    got = gls.token_logprobs(many, t2, top=20)
    ref.check_logprobs(got, ref.logprobs(many, t2, _inv(200, 1, 16), 20), "special, many rows")


def test_logprobs_token_out_of_range(gls):
    x = _logits((1, 1, 2, 100), BF, 1)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    tok = torch.tensor([[[[5, 100], [-7, 2 ** 31 - 1]]]], dtype=torch.int32, device="cuda")
    got = gls.token_logprobs(x, tok, status=status)
    lp = got["logprobs"][0, 0]
    assert lp[0, 1] == -INF and lp[1, 1] == -INF and lp[1, 0] == 0 and lp[0, 0] < 0
    assert int(status.item()) == gls.DEV_BAD_TOKEN


def test_logprobs_peaked_rows(gls):
    """A token that takes nearly all of the mass: log probability and entropy near 0."""
    V = 50000
    x = torch.zeros((3, 1, 1, V), device="cuda")
    x[:, 0, 0, 777] = torch.tensor([20.0, 40.0, 90.0], device="cuda")
    tok = torch.full((3, 1, 1), 777, dtype=torch.int32, device="cuda")
    got = _check(gls, x, tok, 3, what="peaked")
    assert bool((got["entropy"] >= 0).all()) and bool((got["logprobs"] <= 0).all())


def test_logprobs_full_size_row(gls):
    for dtype in (BF, F):
        x = _logits((2, 1, 1, 152064), dtype, 9)
        x[..., -128:] = -INF
        for M in (0, 20, 50):
            _check(gls, x, _tokens((2, 1, 1), 151000, 4), M, what="152064 M=%d" % M)


@pytest.mark.parametrize("dtype,V", [(F, 300007), (BF, 1300003), (F, 1250011), (BF, 2500007)])
def test_logprobs_long_rows(gls, dtype, V):
    """Rows so long that an entry of the selection covers several steps of a warp: few rows, and as many
    (one read again and again) as are scored a warp each."""
    x = _logits((1, 1, 3, V), dtype, V)
    x[0, 0, 2] = x[0, 0, 2].float().sort().values.to(dtype)  # ascending
    tok = _tokens((1, 1, 3), V, 6, none=0.0)
    few = _check(gls, x, tok, 40, what="long rows V=%d %s" % (V, dtype))
    many = gls.token_logprobs(x.expand(800, 1, 3, V), tok.expand(800, 1, 3).contiguous(), top=40)
    for n in ("logprobs", "lse", "entropy", "top_logprobs"):
        tol = 2 * (ref.ENT if n == "entropy" else ref.LSE)
        ref.near(many[n], few[n].double().expand(many[n].shape), tol, "many long rows " + n)
    assert torch.equal(many["top_ids"], few["top_ids"].expand(800, 1, 3, 40))


def test_logprobs_elements_past_32_bits(gls):
    """Row offsets beyond 2^32 elements (8.9 GB of bf16 rows, two of them looked at)."""
    V, B = 152064, 29000
    x = torch.empty((B, 1, 1, V), dtype=BF, device="cuda")
    rows = [0, B - 1]
    for n, r in enumerate(rows):
        x[r] = _logits((1, 1, V), BF, 40 + n)
    view = x.as_strided((2, 1, 1, V), ((B - 1) * V, V, V, 1))
    tok = _tokens((2, 1, 1), V, 8, none=0.0)
    _check(gls, view, tok, 20, what="far rows")
    g = torch.ones((2, 1, 1), device="cuda")
    out = gls.token_logprobs(view, tok)
    back = torch.empty((B, 1, 1, V), dtype=BF, device="cuda")
    bview = back.as_strided((2, 1, 1, V), ((B - 1) * V, V, V, 1))
    gls.token_logprobs_backward(view, tok, out["lse"], grad_logprobs=g, grad_logits=bview)
    want, scale = ref.gradient(view, tok[..., None], _inv(2, 1, 1), g[..., None])
    ref.check_gradient(bview, want, scale, "far rows")


# ---- what a verification emitted ------------------------------------------------------------------
@pytest.mark.parametrize("flags", [0, 1, 2, 3])
@pytest.mark.parametrize("dtype", [F, BF])
def test_emitted_after_verification(gls, dtype, flags):
    B, K, L, V = 9, 4, 3, 3011
    d = _logits((B, K, L, V), F, 11)
    t = torch.empty((B, K, L + 1, V), device="cuda")
    t[:, :, :L] = d + 0.4 * torch.randn(d.shape, generator=_gen(2), device="cuda")
    t[:, :, L] = _logits((B, K, V), F, 13)
    d, t = d.to(dtype), t.to(dtype)
    if flags & gls.NO_BONUS:
        t = t[:, :, :L]
    J = t.shape[2]
    kw = dict(seed=5, inv_temp=0.9)
    tok, _ = gls.draft_sample(d, **kw)
    out = gls.target_sample_verify(t, tok, flags=flags, **kw)
    tau = out["tau"]
    assert int(tau.min()) < int(tau.max())
    for M in (0, 5):
        got = gls.emitted_logprobs(t, out["tokens"], out["accept"], top=M, inv_temp=0.9, flags=flags)
        acc = out["accept"].cpu().numpy()
        rows = torch.empty((B, J, V), dtype=dtype, device="cuda")
        for b in range(B):
            for j in range(J):
                k = 0 if j == 0 else next((k for k in range(K) if acc[b, k, j - 1]), 0)
                rows[b, j] = t[b, k, j]
        live = torch.arange(J, device="cuda")[None] < tau[:, None]
        assert torch.equal(live, out["tokens"] >= 0)
        want = ref.logprobs(rows, out["tokens"][..., None], _inv(B, 1, J, 0.9)[:, 0], M)
        want["logprobs"] = want["logprobs"][..., 0]
        for n in want:
            keep = live if want[n].dim() == 2 else live[..., None]
            want[n] = torch.where(keep, want[n], torch.full_like(want[n], -1 if n == "top_ids" else 0))
        ref.check_logprobs(got, want, "emitted flags=%d M=%d" % (flags, M))


def test_emitted_reads_only_the_rows_it_needs(gls):
    """NaN in every row that no emitted token needs changes nothing, also with 64 drafts and one position."""
    B, K, L, V = 3, 64, 2, 700
    t = _logits((B, K, L + 1, V), F, 3)
    accept = torch.zeros((B, K, L), dtype=torch.uint8, device="cuda")
    accept[0, 40, 0] = accept[0, 63, 0] = accept[0, 63, 1] = 1
    accept[1, 5, 0] = 1
    tok = torch.tensor([[1, 2, 3], [4, 5, -1], [6, -1, -1]], dtype=torch.int32, device="cuda")
    got = gls.emitted_logprobs(t, tok, accept, top=3)
    x = torch.full_like(t, float("nan"))
    for b, k, j in [(0, 0, 0), (0, 40, 1), (0, 63, 2), (1, 0, 0), (1, 5, 1), (2, 0, 0)]:
        x[b, k, j] = t[b, k, j]
    again = gls.emitted_logprobs(x, tok, accept, top=3)
    for n in got:
        assert torch.equal(got[n], again[n]), n
    one = gls.emitted_logprobs(t[:, :, :1], tok[:, :1].contiguous(), None, top=3)
    assert torch.equal(one["logprobs"][:, 0], got["logprobs"][:, 0])


# ---- gradient of log probabilities --------------------------------------------------------------
def _grads(shape, G, M, seed):
    g = _gen(seed)
    return dict(g_lp=torch.randn(shape + (G,), generator=g, device="cuda") if G else None,
                g_lse=torch.randn(shape, generator=g, device="cuda"),
                g_ent=0.3 * torch.randn(shape, generator=g, device="cuda"),
                g_top=torch.randn(shape + (M,), generator=g, device="cuda") if M else None)


def _check_grad(gls, x, tok, M, which, inv_temp=1.0, per=None, grad_logits=None, what="", seed=3):
    B, K, J, V = x.shape
    inv = _inv(B, K, J, inv_temp, per)
    out = dict(logprobs=torch.empty(tok.shape, device="cuda"), lse=torch.empty((B, K, J), device="cuda"),
               lse_tail=torch.empty((B, K, J), device="cuda"), entropy=torch.empty((B, K, J), device="cuda"))
    if M:
        out["top_ids"] = torch.empty((B, K, J, M), dtype=torch.int32, device="cuda")
        out["top_logprobs"] = torch.empty((B, K, J, M), device="cuda")
    gls.token_logprobs(x, tok, top=M, inv_temp=inv_temp, inv_temp_per_draft=per, out=out)
    t4 = tok if tok.dim() == 4 else tok[..., None]
    g = {n: v if n in which else None for n, v in _grads((B, K, J), t4.shape[-1], M, seed).items()}
    got = gls.token_logprobs_backward(
        x, tok, out["lse"], entropy=out["entropy"], lse_tail=out["lse_tail"], top_ids=out.get("top_ids"),
        grad_logprobs=None if g["g_lp"] is None else g["g_lp"].view(tok.shape).contiguous(), grad_lse=g["g_lse"],
        grad_entropy=g["g_ent"], grad_top_logprobs=g["g_top"], inv_temp=inv_temp, inv_temp_per_draft=per,
        grad_logits=grad_logits)
    want, scale = ref.gradient(x, t4, inv, top_ids=out.get("top_ids"), **g)
    assert not bool(torch.isnan(got).any()), what
    ref.check_gradient(got, want, scale, what)
    return got


ALL = ("g_lp", "g_lse", "g_ent", "g_top")


@pytest.mark.parametrize("dtype", [F, BF])
@pytest.mark.parametrize("V", [1, 2, 15, 17, 511, 2049, 4099, 16385, 40001])
def test_gradient_sizes(gls, dtype, V):
    x = _logits((2, 3, 2, V), dtype, V)
    tok = _tokens((2, 3, 2), V, V)
    for M, which in ((0, ("g_lp",)), (0, ("g_lp", "g_ent")), (5, ALL), (0, ("g_lse",)), (3, ("g_top",))):
        _check_grad(gls, x, tok, M, which, 1.25, what="V=%d %s %s" % (V, which, dtype))


@pytest.mark.parametrize("dtype", [F, BF])
def test_gradient_several_tokens(gls, dtype):
    """The same token given several times, among the alternatives too, and tokens that are none."""
    B, K, J, V = 2, 2, 2, 3000
    x = _logits((B, K, J, V), dtype, 5)
    tok = _tokens((B, K, J, 40), V, 4)
    tok[0, 0, 0] = int(x[0, 0, 0].float().argmax())
    tok[0, 1, 0, ::2] = 9
    tok[1, 0, 0] = -1
    _check_grad(gls, x, tok, 50, ALL, per=[0.5, 2.0], what="several tokens")


@pytest.mark.parametrize("dtype", [F, BF])
def test_gradient_strides(gls, dtype):
    base = _logits((2, 3, 4, 3040), dtype, 6)
    for off, goff in ((1, 1), (3, 0), (0, 5), (16, 16), (7, 23)):
        x = base[..., off:off + 3000]
        out = torch.full((2, 3, 4, 3040), 7.0, dtype=dtype, device="cuda")
        view = out[..., goff:goff + 3000]
        _check_grad(gls, x, _tokens((2, 3, 4), 3000, off), 3, ALL, grad_logits=view, what="offsets %d %d" % (off, goff))
        view.fill_(7.0)
        assert bool((out == 7.0).all())  # nothing beside the rows was written
    x = base[:, :1].expand(2, 5, 4, 3040)
    _check_grad(gls, x, _tokens((2, 5, 4), 3040, 2), 3, ALL, what="shared rows")
    _check_grad(gls, base.permute(2, 1, 0, 3), _tokens((4, 3, 2), 3040, 2), 3, ALL, what="permuted")


@pytest.mark.parametrize("dtype", [F, BF])
@pytest.mark.parametrize("V", [40, 2100, 20011])
def test_gradient_special_rows(gls, dtype, V):
    x = _special(dtype, V).view(2, 2, 4, V)
    tok = _tokens((2, 2, 4, 3), V, 1)
    tok[..., 0] = V // 2
    for which in (("g_lp",), ALL):
        _check_grad(gls, x, tok, 20, which, what="special V=%d %s" % (V, which))


@pytest.mark.parametrize("dtype", [F, BF])
@pytest.mark.parametrize("inv_temp", [1e-20, 1e-6, 3e3, 1e9, 1e20])
def test_extreme_temperatures(gls, dtype, inv_temp):
    """From a uniform law to one token that takes all, forward and backward."""
    x = _logits((2, 1, 2, 3001), dtype, 14) + (0 if dtype == BF else 40.0)
    x[1, 0, 1, 7:9] = -INF
    tok = _tokens((2, 1, 2), 3001, 15, none=0.0)
    tok[0, 0, 0] = int(x[0, 0, 0].float().argmax())
    _check(gls, x, tok, 5, inv_temp, what="inv_temp %g %s" % (inv_temp, dtype))
    for which in (("g_lp",), ALL):
        _check_grad(gls, x, tok, 5, which, inv_temp, what="inv_temp %g %s" % (inv_temp, dtype))


def test_gradient_against_differences(gls):
    """Central differences of the 64-bit formula, in a random direction."""
    B, K, J, V = 2, 1, 2, 200
    x = _logits((B, K, J, V), F, 8, sd=1.5)
    tok = _tokens((B, K, J), V, 8, none=0.0)
    g = _grads((B, K, J), 1, 0, 8)
    out = gls.token_logprobs(x, tok, inv_temp=0.8)
    got = gls.token_logprobs_backward(x, tok, out["lse"], entropy=out["entropy"], grad_logprobs=g["g_lp"][..., 0].contiguous(),
                                      grad_lse=g["g_lse"], grad_entropy=g["g_ent"], inv_temp=0.8).double()
    inv = _inv(B, K, J, 0.8)
    d = torch.randn(x.shape, generator=_gen(9), device="cuda", dtype=torch.float64)

    def loss(y):
        o = ref.logprobs(y, tok[..., None], inv, 0)
        return float((o["logprobs"] * g["g_lp"].double()).sum() + (o["lse"] * g["g_lse"].double()).sum()
                     + (o["entropy"] * g["g_ent"].double()).sum())
    h = 1e-4
    slope = (loss(x.double() + h * d) - loss(x.double() - h * d)) / (2 * h)
    # differences of second order: h^2 times third derivatives (below 10), and 1e-15 / h of rounding;
    # the gradient itself is fp32: 3e-5 of the sum of |gradient| |d|
    assert abs(slope - float((got * d).sum())) <= 1e-6 + 3e-5 * float((got.abs() * d.abs()).sum())


def test_autograd_of_logprobs(gls):
    B, K, J, V, M = 2, 2, 3, 1501, 4
    x = _logits((B, K, J, V), F, 21).requires_grad_()
    tok = _tokens((B, K, J), V, 22)
    o = gls.token_logprobs(x, tok, top=M, inv_temp=0.7)
    assert not o["top_ids"].requires_grad
    loss = -(o["logprobs"].mean()) + 1e-2 * o["lse"].square().mean() - 0.1 * o["entropy"].mean() + o["top_logprobs"].sum() * 0.01
    loss.backward()
    y = x.detach().double().requires_grad_()
    lp = torch.log_softmax(y * ref.f32(0.7), -1)
    live = (tok >= 0).double()
    lse = torch.logsumexp(y * ref.f32(0.7), -1)
    given = lp.gather(-1, tok.long().clamp(min=0)[..., None])[..., 0] * live
    l2 = -(given.mean()) + 1e-2 * lse.square().mean() - 0.1 * (-(lp.exp() * lp).sum(-1)).mean() + \
        lp.gather(-1, o["top_ids"].long()).sum() * 0.01
    l2.backward()
    n = B * K * J
    a = 1 / n + 0.02 * lse.abs()[..., None].detach() / n + 0.01 * M
    p = lp.exp().detach()
    scale = 0.7 * p * (2.8e-5 * (a + 0.1 / n * (lp.detach().abs() + 8)) + ref.ENT) + 4 * ref.U
    ref.near(x.grad, y.grad, scale + ref.U * y.grad.abs(), "autograd")
    # an expanded input: the gradients of the shared row are added by autograd
    z = _logits((1, 1, 1, V), F, 30).requires_grad_()
    gls.token_logprobs(z.expand(2, 3, 1, V), _tokens((2, 3, 1), V, 31, none=0.0))["logprobs"].sum().backward()
    assert z.grad.shape == z.shape and abs(float(z.grad.double().sum())) < 1e-3
    with pytest.raises(gls.GlsError):
        gls.token_logprobs(x, tok, out=dict(logprobs=o["logprobs"].detach(), lse=o["lse"].detach()))


# ---- embedding ----------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [F, BF])
@pytest.mark.parametrize("V,D,N", [(1, 1, 1), (5, 8, 3), (100, 16, 1000), (37, 33, 70), (3000, 1024, 17),
                                   (500, 4096, 300), (20, 8200, 9), (1000, 7, 4097), (300, 504, 77), (300, 512, 77),
                                   (300, 520, 77), (300, 1016, 50)])
def test_embedding(gls, dtype, V, D, N):
    table = torch.randn((V, D), generator=_gen(V), device="cuda").to(dtype)
    tok = _tokens((N,), V, N)
    for scale in (1.0, 0.3):
        got = gls.embed_tokens(table, tok, scale=scale)
        want = table.double()[tok.long().clamp(min=0)] * ref.f32(scale) * (tok >= 0).double()[:, None]
        # the product is rounded to fp32 and then to the output's type
        tol = (ref.HALF[dtype] + 2 * ref.U) * want.abs()
        if scale == 1.0:
            tol = tol * 0
        ref.near(got, want, tol, "embedding %s" % scale)


@pytest.mark.parametrize("dtype", [F, BF])
def test_embedding_strides_shapes_and_bad_tokens(gls, dtype):
    big = torch.randn((50, 100), generator=_gen(1), device="cuda").to(dtype)
    tok = _tokens((2, 3, 4), 50, 2)
    for off in (0, 1, 8):
        t = big[:, off:off + 64]
        out = torch.full((2, 3, 4, 80), 3.0, dtype=dtype, device="cuda")
        got = gls.embed_tokens(t, tok, out=out[..., :64])
        assert torch.equal(got, t[tok.long().clamp(min=0)] * (tok >= 0)[..., None])
        assert bool((out[..., 64:] == 3.0).all())
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    bad = torch.tensor([3, 50, -5, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    got = gls.embed_tokens(big, bad, status=status)
    assert torch.equal(got[0], big[3]) and bool((got[1:] == 0).all()) and int(status.item()) == gls.DEV_BAD_TOKEN
    assert gls.embed_tokens(big, bad[:0]).shape == (0, 100)
    nan = torch.full((3, 8), float("nan"), dtype=dtype, device="cuda")  # zeros are zeros, not NaN * 0
    assert bool((gls.embed_tokens(nan, bad[2:3], scale=2.0) == 0).all())


def _skewed(N, V, seed, none=0.05):
    """Tokens whose frequency falls off as 1 / rank, with a share of none."""
    r = torch.exp(torch.rand(N, generator=_gen(seed), device="cuda", dtype=torch.float64) * torch.log(torch.tensor(float(V + 1))))
    t = (r.long().clamp(1, V) - 1) * 7919 % V
    return torch.where(torch.rand(N, generator=_gen(seed + 1), device="cuda") < none, torch.full_like(t, -1), t).to(torch.int32)


def _embed_grad_ref(g, tok, V, scale):
    live = tok >= 0
    t = tok.long()[live]
    x = g.double().reshape(tok.numel(), -1)[live]
    s = torch.zeros((V, x.shape[1]), dtype=torch.float64, device="cuda").index_add_(0, t, x)
    a = torch.zeros((V, x.shape[1]), dtype=torch.float64, device="cuda").index_add_(0, t, x.abs())
    n = torch.zeros(V, dtype=torch.float64, device="cuda").index_add_(0, t, torch.ones_like(t, dtype=torch.float64))
    # n additions and the scaling, one half step of fp32 of the running sum each
    return s * ref.f32(scale), (n[:, None] + 2) * ref.U * a * abs(scale)


@pytest.mark.parametrize("dtype", [F, BF])
@pytest.mark.parametrize("N,V,D", [(1, 1, 1), (3, 5, 8), (64, 7, 40), (1000, 50, 33), (4096, 30000, 64), (4097, 600, 24),
                                   (9000, 152064, 16), (20000, 300, 264), (50000, 1 << 20, 8), (5000, 3, 1032),
                                   (300, 2000, 4104), (16384, 700, 16), (16385, 70000, 16), (20000, 40000, 1024),
                                   (32768, 900, 8), (32769, 900, 8), (150000, 5000, 16),
                                   (400000, 200, 8), (70000, 3000000, 8)])
def test_embedding_gradient(gls, dtype, N, V, D):
    g = torch.randn((N, D), generator=_gen(N), device="cuda").to(dtype)
    tok = _skewed(N, V, N)
    want, scale = _embed_grad_ref(g, tok, V, 0.3)
    got = gls.embed_tokens_backward(g, tok, V, scale=0.3)
    ref.check_gradient(got, want, scale, "embedding gradient N=%d V=%d D=%d %s" % (N, V, D, dtype))
    again = gls.embed_tokens_backward(g, tok, V, scale=0.3)
    assert torch.equal(got, again)
    # fp32 sums of any input type, added to what is there; other rows are left as they are
    acc = torch.randn((V, D), generator=_gen(7), device="cuda")
    before = acc.clone()
    gls.embed_tokens_backward(g, tok, V, scale=0.3, grad_table=acc, accumulate=True)
    touched = torch.zeros(V, dtype=torch.bool, device="cuda")
    touched[tok.long()[tok >= 0]] = True
    assert torch.equal(acc[~touched], before[~touched])
    ref.check_gradient(acc, before.double() + want, scale + ref.U * want.abs(), "accumulated")


def _odd(rows, D, off, pad, dtype, fill):
    """(buffer, its rows [rows, D]: `off` elements in, `pad` between them, nothing behind the last)"""
    buf = torch.full((off + rows * (D + pad) - pad,), fill, dtype=dtype, device="cuda")
    return buf, buf.as_strided((rows, D), (D + pad, 1), off)


def _outside(buf, view):
    out = torch.ones_like(buf, dtype=torch.bool)
    out.as_strided(view.shape, view.stride(), view.storage_offset())[:] = False
    return buf[out]


ODD = [1, 2, 3, 5, 7, 8, 9, 15, 17, 31, 40, 63, 65, 129, 511, 515, 1002, 2051, 2283, 4101]


@pytest.mark.parametrize("dtype", [F, BF])
@pytest.mark.parametrize("D", ODD)
def test_embedding_of_odd_rows(gls, dtype, D):
    V, N = 37, 301
    tok = _tokens((N,), V, D)
    tok[0], tok[1], tok[2], tok[N - 1] = V - 1, 0, -1, V - 1
    for n, (off, pad, ooff, opad) in enumerate([(0, 0, 0, 0), (1, 0, 0, 0), (0, 0, 1, 0), (3, 1, 5, 2), (7, 8, 2, 0), (8, 0, 3, 5)]):
        buf, table = _odd(V, D, off, pad, dtype, float("nan"))  # what lies between the rows is not used
        table.copy_(torch.randn((V, D), generator=_gen(D + n), device="cuda"))
        obuf, out = _odd(N, D, ooff, opad, dtype, 3.0)
        for scale in (1.0, -0.3):
            gls.embed_tokens(table, tok, scale=scale, out=out)
            want = table.double()[tok.long().clamp(min=0)] * ref.f32(scale) * (tok >= 0).double()[:, None]
            ref.near(out, want, (ref.HALF[dtype] + 2 * ref.U) * want.abs() * (scale != 1.0), "D=%d %d" % (D, n))
            assert bool((_outside(obuf, out) == 3.0).all())


@pytest.mark.parametrize("dtype,out_dtype", [(F, F), (BF, BF), (BF, F)])
@pytest.mark.parametrize("D", ODD)
def test_embedding_gradient_of_odd_rows(gls, dtype, out_dtype, D):
    for n, (N, V, off, pad, ooff, opad) in enumerate([(300, 40, 0, 0, 0, 0), (700, 900, 1, 0, 3, 0), (3000, 5, 3, 2, 1, 1),
                                                      (20000, 70, 0, 1, 2, 0), (40, 3000, 5, 0, 0, 7)]):
        if N * D > 1 << 23:
            continue
        _, g = _odd(N, D, off, pad, dtype, float("nan"))
        g.copy_(torch.randn((N, D), generator=_gen(D + n), device="cuda"))
        tok = _skewed(N, V, D + n)
        want, scale = _embed_grad_ref(g, tok, V, 0.3)
        buf, out = _odd(V, D, ooff, opad, out_dtype, 3.0)
        gls.embed_tokens_backward(g, tok, V, scale=0.3, grad_table=out)
        ref.check_gradient(out, want, scale, "D=%d %d" % (D, n))
        assert bool((_outside(buf, out) == 3.0).all())
        first = out.clone()
        gls.embed_tokens_backward(g, tok, V, scale=0.3, grad_table=out, accumulate=True)
        # the sum is rounded to the output's type, which check_gradient counts
        ref.check_gradient(out, first.double() + want, scale + ref.U * (first.double().abs() + want.abs()), "accumulated %d" % n)
        touched = torch.zeros(V, dtype=torch.bool, device="cuda")
        touched[tok.long()[tok >= 0]] = True
        assert torch.equal(out[~touched], first[~touched]) and bool((_outside(buf, out) == 3.0).all())


@pytest.mark.parametrize("dtype", [F, BF])
def test_embedding_gradient_special(gls, dtype):
    V, D = 100, 48
    g = torch.randn((6000, D), generator=_gen(1), device="cuda").to(dtype)
    one = torch.full((6000,), 17, dtype=torch.int32, device="cuda")          # one token all over
    want, scale = _embed_grad_ref(g, one, V, 1.0)
    ref.check_gradient(gls.embed_tokens_backward(g, one, V), want, scale, "one token")
    none = torch.full((6000,), -1, dtype=torch.int32, device="cuda")         # no token at all
    assert bool((gls.embed_tokens_backward(g, none, V) == 0).all())
    empty = gls.embed_tokens_backward(g[:0], none[:0], V)
    assert empty.shape == (V, D) and bool((empty == 0).all())
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    for n in (100, 6000):
        bad = torch.full((n,), V, dtype=torch.int32, device="cuda")          # outside the table
        status.zero_()
        assert bool((gls.embed_tokens_backward(g[:n], bad, V, status=status) == 0).all())
        assert int(status.item()) == gls.DEV_BAD_TOKEN
    # rows of padding hold garbage that must not reach the sums
    tok = _skewed(6000, V, 3, none=0.3)
    dirty = g.clone()
    dirty[tok < 0] = float("nan")
    assert torch.equal(gls.embed_tokens_backward(dirty, tok, V), gls.embed_tokens_backward(g, tok, V))
    # views: wide rows, an offset, an expanded gradient, a table that is a view
    wide = torch.randn((6000, 100), generator=_gen(2), device="cuda").to(dtype)
    for off in (0, 1, 8):
        v = wide[:, off:off + D]
        out = torch.full((V, D + 5), 9.0, dtype=dtype, device="cuda")
        want, scale = _embed_grad_ref(v, tok, V, 2.0)
        ref.check_gradient(gls.embed_tokens_backward(v, tok, V, scale=2.0, grad_table=out[:, :D]), want, scale, "view")
        assert bool((out[:, D:] == 9.0).all())
    e = g[:1].expand(6000, D)
    want, scale = _embed_grad_ref(e, tok, V, 1.0)
    ref.check_gradient(gls.embed_tokens_backward(e, tok, V), want, scale, "expanded")


def test_embedding_gradient_against_differences(gls):
    V, D, N = 11, 6, 40
    table = torch.randn((V, D), generator=_gen(3), device="cuda", requires_grad=True)
    tok = _tokens((N,), V, 4)
    w = torch.randn((N, D), generator=_gen(5), device="cuda")
    (gls.embed_tokens(table, tok, scale=1.5) * w).sum().backward()
    live = (tok >= 0).double()[:, None]

    def loss(t):
        return float((t[tok.long().clamp(min=0)] * 1.5 * live * w.double()).sum())
    d = torch.randn((V, D), generator=_gen(6), device="cuda", dtype=torch.float64)
    t0 = table.detach().double()
    slope = (loss(t0 + d) - loss(t0 - d)) / 2  # linear: exact up to rounding
    assert abs(slope - float((table.grad.double() * d).sum())) <= 1e-9 + 50 * ref.U * float((table.grad.abs().double() * d.abs()).sum())


# ---- together -----------------------------------------------------------------------------------
def test_a_drafter_learns_from_its_tokens(gls):
    """Embedding, a layer, log probabilities, and the gradients of table and weights, against 64 bits."""
    V, D, B, L = 700, 64, 5, 6
    gen = _gen(12)
    table = (0.2 * torch.randn((V, D), generator=gen, device="cuda")).requires_grad_()
    head = (0.2 * torch.randn((D, V), generator=gen, device="cuda")).requires_grad_()
    tok = _tokens((B, 1, L + 1), V, 13, none=0.1)
    x, y = tok[:, :, :-1].contiguous(), tok[:, :, 1:].contiguous()
    h = gls.embed_tokens(table, x, scale=D ** 0.5)
    o = gls.token_logprobs(torch.tanh(h) @ head, y, inv_temp=1.25)
    n = int((y >= 0).sum())
    loss = -o["logprobs"].sum() / n - 0.01 * o["entropy"].mean()
    loss.backward()
    t2, h2 = table.detach().double().requires_grad_(), head.detach().double().requires_grad_()
    e = t2[x.long().clamp(min=0)] * (x >= 0).double()[..., None] * D ** 0.5
    z = torch.log_softmax(torch.tanh(e) @ h2 * 1.25, -1)
    lp = z.gather(-1, y.long().clamp(min=0)[..., None])[..., 0] * (y >= 0).double()
    l2 = -lp.sum() / n - 0.01 * (-(z.exp() * z).sum(-1)).mean()
    l2.backward()
    assert abs(float(loss.detach()) - float(l2.detach())) < 1e-4
    for a, b in ((table.grad, t2.grad), (head.grad, h2.grad)):
        # matrix products of fp32 numbers of 64 and 700 terms around the operators: 1e-4 of the largest
        assert float((a.double() - b).abs().max()) <= 1e-4 * float(b.abs().max())


def test_serving_step_with_answers(gls):
    """Draft, verify, then the emitted tokens' log probabilities and the next inputs, on one stream that
    is not the default one, captured into a graph and replayed on new logits."""
    B, K, L, V, D = 4, 3, 2, 5003, 40
    dev = "cuda"
    d, t = torch.empty((B, K, L, V), device=dev), torch.empty((B, K, L + 1, V), device=dev)
    table = torch.randn((V, D), generator=_gen(1), device=dev)

    def fill(seed):
        d.copy_(_logits((B, K, L, V), F, seed))
        t.copy_(_logits((B, K, L + 1, V), F, seed + 5))
        t[:, :, :L].copy_(d + 0.2)

    def step():
        tok, _ = gls.draft_sample(d, seed=3)
        out = gls.target_sample_verify(t, tok, seed=3)
        o = gls.emitted_logprobs(t, out["tokens"], out["accept"], top=4)
        return out, o, gls.embed_tokens(table, out["tokens"], scale=2.0)

    fill(50)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for seed in (50, 60):
        fill(seed)
        torch.cuda.synchronize()
        want = step()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(want[0]["tokens"], held[0]["tokens"])
        for n in want[1]:
            assert torch.equal(want[1][n], held[1][n]), n
        assert torch.equal(want[2], held[2])


@pytest.mark.parametrize("fused", [False, True])
def test_spec_step_reports_on_the_emitted_tokens(gls, fused):
    """The pipeline's step with answers and next inputs, and as a captured graph on refilled logits."""
    from paper_2506_05632_b200 import pipeline

    B, K, L, V, D = 5, 3, 2, 4001, 24
    t = _logits((B, K, L + 1, V), BF, 90)
    d = (t[:, :, :L].float() + 0.5 * torch.randn((B, K, L, V), generator=_gen(91), device="cuda")).to(BF)
    table = torch.randn((V, D), generator=_gen(92), device="cuda").to(BF)
    buf = pipeline.StepBuffers(B, K, L, V, top=6, table=table, table_scale=2.0)
    plain = pipeline.StepBuffers(B, K, L, V)
    kw = dict(inv_temp=0.8, seed=7, fused=fused)

    def check():
        want = pipeline.spec_step(d, t, plain, **kw)
        for n in want:
            assert torch.equal(buf.out[n], want[n]), n
        answers = gls.emitted_logprobs(t, want["tokens"], want["accept"], top=6, inv_temp=0.8)
        for n in answers:
            assert torch.equal(buf.answers[n], answers[n]), n
        live = (want["tokens"] >= 0)[..., None]
        assert torch.equal(buf.inputs, table[want["tokens"].long().clamp(min=0)] * 2.0 * live)
    pipeline.spec_step(d, t, buf, **kw)
    check()
    graph = pipeline.GraphedStep(d, t, buf, **kw)
    t.copy_(_logits((B, K, L + 1, V), BF, 95))
    graph.replay()
    torch.cuda.synchronize()
    check()
    assert int(buf.status.item()) == 0


def test_backward_in_a_graph(gls):
    """The binding's backward functions captured while an eager graph of the same leaf is alive; the
    differentiable form refuses the capture."""
    B, K, J, V, D, N = 2, 2, 2, 3001, 24, 5000
    x = _logits((B, K, J, V), BF, 1)
    leaf = x.clone().requires_grad_()
    tok = _tokens((B, K, J), V, 2)
    alive = gls.token_logprobs(leaf, tok)  # an eager graph of this leaf
    g = torch.randn((B, K, J), generator=_gen(3), device="cuda")
    go, tk = torch.randn((N, D), generator=_gen(4), device="cuda"), _skewed(N, 300, 5)

    def step():
        o = gls.token_logprobs(x, tok, top=3)
        return (gls.token_logprobs_backward(x, tok, o["lse"], entropy=o["entropy"], grad_logprobs=g, grad_entropy=g),
                gls.embed_tokens_backward(go, tk, 300))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        with pytest.raises(gls.GlsError, match="captured"):
            gls.token_logprobs(leaf, tok)
        held = step()
    x.copy_(_logits((B, K, J, V), BF, 70))
    go.mul_(-0.5)
    want = step()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(held[0], want[0]) and torch.equal(held[1], want[1])
    alive["logprobs"].sum().backward()
    assert leaf.grad is not None


def test_two_streams_and_a_shared_workspace(gls):
    """Calls on two streams with workspaces of their own run side by side; two calls that share one
    are ordered by their stream.  A workspace may hold anything on entry."""
    V, M = 40000, 20
    x = [_logits((2, 2, 2, V), BF, 80 + i) for i in range(4)]
    tok = _tokens((2, 2, 2), V, 3)
    want = [gls.token_logprobs(a, tok, top=M) for a in x]
    go = [torch.randn((7000, 64), generator=_gen(i), device="cuda") for i in range(4)]
    tk = [_skewed(7000, 900, i) for i in range(4)]
    wantg = [gls.embed_tokens_backward(go[i], tk[i], 900) for i in range(4)]
    torch.cuda.synchronize()
    ne = gls.embed_tokens_backward_workspace_bytes(7000, 900, 64)
    streams = [torch.cuda.Stream() for _ in range(2)]
    we = [torch.full((ne,), 0xA5, dtype=torch.uint8, device="cuda") for _ in range(2)]
    torch.cuda.synchronize()
    got, gotg = [None] * 4, [None] * 4
    for i in range(4):
        with torch.cuda.stream(streams[i % 2]):
            got[i] = gls.token_logprobs(x[i], tok, top=M)
            gotg[i] = gls.embed_tokens_backward(go[i], tk[i], 900, workspace=we[i % 2])
    torch.cuda.synchronize()
    for i in range(4):
        for k in want[i]:
            assert torch.equal(got[i][k], want[i][k]), (i, k)
        assert torch.equal(gotg[i], wantg[i])


def test_refusals_of_the_binding(gls):
    x = _logits((1, 2, 3, 100), BF, 1)
    tok = _tokens((1, 2, 3), 100, 1)
    ok = gls.token_logprobs(x, tok, top=3)
    bad = [lambda: gls.token_logprobs(x.half(), tok), lambda: gls.token_logprobs(x, tok.long()),
           lambda: gls.token_logprobs(x, tok[:, :1]), lambda: gls.token_logprobs(x, tok, top=257),
           lambda: gls.token_logprobs(x, tok, top=-1), lambda: gls.token_logprobs(x, tok, inv_temp=0.0),
           lambda: gls.token_logprobs(x, tok, inv_temp_per_draft=[1.0]),
           lambda: gls.token_logprobs(x.transpose(2, 3), tok),
           lambda: gls.token_logprobs(x, tok.expand(1, 2, 3).transpose(1, 2)),
           lambda: gls.token_logprobs(x, torch.zeros((1, 2, 3, 65), dtype=torch.int32, device="cuda")),
           lambda: gls.embed_tokens_backward(x[0, 0], tok.view(6)[:3], 9,
                                             workspace=torch.empty(8, dtype=torch.uint8, device="cuda")),
           lambda: gls.emitted_logprobs(x, tok[:, 0].contiguous(), None),
           lambda: gls.token_logprobs_backward(x, tok, ok["lse"], grad_entropy=ok["lse"]),
           lambda: gls.token_logprobs_backward(x, tok, ok["lse"], grad_top_logprobs=ok["top_logprobs"]),
           lambda: gls.token_logprobs_backward(x, tok, ok["lse"].double()),
           lambda: gls.token_logprobs_backward(x, tok, ok["lse"], grad_logits=x),
           lambda: gls.token_logprobs_backward(x, tok, ok["lse"], grad_logits=x[:, :1].clone().expand(1, 2, 3, 100)),
           lambda: gls.embed_tokens(x[0, 0].half(), tok), lambda: gls.embed_tokens(x[0, 0].t(), tok),
           lambda: gls.embed_tokens(x[0, 0], tok.long()),
           lambda: gls.embed_tokens(x[0, 0], tok, out=torch.empty((1, 2, 3, 50), dtype=BF, device="cuda")),
           lambda: gls.embed_tokens_backward(x[0, 0], tok.view(6)[:2], 9),
           lambda: gls.embed_tokens_backward(x[0, 0], tok.view(6)[:3], 9, accumulate=True),
           lambda: gls.embed_tokens_backward(x[0, 0].float(), tok.view(6)[:3], 9,
                                             grad_table=torch.empty((9, 100), dtype=BF, device="cuda"))]
    for n, f in enumerate(bad):
        with pytest.raises(gls.GlsError):
            f()
            raise AssertionError("call %d was accepted" % n)


class _Declines:
    """Stands in for the compiled module: every call goes the general way."""

    def __getattr__(self, name):
        return lambda *a: None


def _same(a, b):
    if isinstance(a, dict):
        assert set(a) == set(b)
        for n in a:
            _same(a[n], b[n])
        return
    assert a.dtype == b.dtype and a.shape == b.shape and a.is_contiguous()
    assert torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


@pytest.mark.parametrize("dtype", [F, BF])
def test_both_ways_of_a_call(gls, dtype, monkeypatch):
    """The compiled module and the binding's own path: the same tensors, the same errors."""
    x = _logits((2, 3, 4, 1030), dtype, 1)[..., :1021]  # rows that start off a 16-byte boundary
    tok, many = _tokens((2, 3, 4), 1021, 2), _tokens((2, 3, 4, 5), 1021, 3)
    bad = _tokens((2, 3, 4), 2000, 4)
    d = _tokens((2, 3, 3), 1021, 5, none=0)
    v = gls.target_sample_verify(x, d, inv_temp=1.25, seed=7)
    table = torch.randn(77, 24, generator=_gen(6), device="cuda").to(dtype)
    g = torch.randn(2, 3, 4, 24, generator=_gen(7), device="cuda").to(dtype)
    gl = torch.randn(2, 3, 4, generator=_gen(8), device="cuda")

    def all_calls():
        status = [torch.zeros(1, dtype=torch.int32, device="cuda") for _ in range(4)]
        f = gls.token_logprobs(x, tok, top=7, inv_temp=2, status=status[0])
        out = [f, gls.token_logprobs(x, many, 0, 0.5, None, False), gls.token_logprobs(x, bad, 300 - 44, status=status[1]),
               gls.token_logprobs(x, many[..., :0].contiguous()), gls.token_logprobs(x, None, 3),
               gls.emitted_logprobs(x, v["tokens"], v["accept"], top=4, inv_temp=1.25, status=status[2]),
               gls.token_logprobs_backward(x, tok, f["lse"], entropy=f["entropy"], top_ids=f["top_ids"], grad_logprobs=gl,
                                           grad_entropy=gl, grad_top_logprobs=f["top_logprobs"], inv_temp=2),
               gls.embed_tokens(table, bad % 90, 3, status=status[3]), gls.embed_tokens(table[:, :7], tok % 77, 1.5),
               gls.embed_tokens(table, tok[:0]), gls.embed_tokens_backward(g, tok % 77, 77, 1.5),
               gls.embed_tokens_backward(g[:0], tok[:0], 77), gls.embed_tokens_backward(g[..., :1], tok % 77, 77)]
        return out + status

    def errors():
        z = torch.zeros
        calls = [lambda: gls.token_logprobs(x, tok, inv_temp=0.0), lambda: gls.token_logprobs(x, tok, inv_temp=float("nan")),
                 lambda: gls.token_logprobs(x, tok, inv_temp=1 << 2000), lambda: gls.token_logprobs(x, tok, top=-1),
                 lambda: gls.token_logprobs(x, tok, top=1 << 70), lambda: gls.token_logprobs(x, tok.long()),
                 lambda: gls.token_logprobs(x, tok.cpu()), lambda: gls.token_logprobs(x, tok[:1]),
                 lambda: gls.token_logprobs(x[..., ::2], tok), lambda: gls.token_logprobs(x.half(), tok),
                 lambda: gls.token_logprobs(x[0], tok), lambda: gls.token_logprobs(x[..., :0], tok),
                 lambda: gls.token_logprobs(x[:0], tok[:0]), lambda: gls.token_logprobs(x, tok, status=z(2).int().cuda()),
                 lambda: gls.token_logprobs(x, tok[..., None].expand(2, 3, 4, 65).contiguous()),
                 lambda: gls.token_logprobs(x[:1, :1, :1].expand(2 ** 31, 1, 1, 1021), tok),
                 lambda: gls.emitted_logprobs(x, v["tokens"], v["accept"][:, :, :2]),
                 lambda: gls.emitted_logprobs(x, v["tokens"].t(), v["accept"]),
                 lambda: gls.emitted_logprobs(x, v["tokens"], v["accept"], flags=64),
                 lambda: gls.token_logprobs_backward(x, tok, gl, grad_entropy=gl),
                 lambda: gls.token_logprobs_backward(x, tok, None, grad_logprobs=gl),
                 lambda: gls.token_logprobs_backward(x, tok, gl, grad_logprobs=gl.double()),
                 lambda: gls.embed_tokens(table, tok, scale=float("inf")), lambda: gls.embed_tokens(table.t(), tok),
                 lambda: gls.embed_tokens(table.cpu(), tok), lambda: gls.embed_tokens(table, tok.cpu()),
                 lambda: gls.embed_tokens_backward(g, tok[:1], 77), lambda: gls.embed_tokens_backward(g, tok, 0),
                 lambda: gls.embed_tokens_backward(g, tok, 77, scale=float("nan"))]
        names = []
        for i, c in enumerate(calls):
            with pytest.raises(Exception) as e:
                c()
                pytest.fail("call %d was not refused" % i)
            names.append((e.type, str(e.value)))
        return names

    got, bad_calls = all_calls(), errors()
    monkeypatch.setattr(gls.binding, "_calls", _Declines())
    want, same_calls = all_calls(), errors()
    for a, b in zip(got, want):
        _same(a, b)
    assert bad_calls == same_calls


def test_calls_from_two_threads(gls):
    """Each thread on its own stream: the calls let other threads run, and keep to their stream."""
    import threading

    x = _logits((4, 2, 3, 5000), BF, 1)
    tok = [_tokens((4, 2, 3), 5000, s) for s in (2, 3)]
    want = [gls.token_logprobs(x, t, top=5) for t in tok]
    torch.cuda.synchronize()
    got, fail = [[], []], []

    def work(i):
        try:
            s = torch.cuda.Stream()
            with torch.cuda.stream(s):
                for _ in range(50):
                    got[i].append(gls.token_logprobs(x, tok[i], top=5))
            s.synchronize()
        except Exception as e:  # pragma: no cover
            fail.append(e)

    ts = [threading.Thread(target=work, args=(i,)) for i in (0, 1)]
    [t.start() for t in ts]
    [t.join() for t in ts]
    assert not fail
    for i in (0, 1):
        assert len(got[i]) == 50
        for r in got[i]:
            _same(r, want[i])
