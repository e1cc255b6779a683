"""Plain 64-bit forms of the operators next to the sampler, and the tolerances of their tests.

Tolerances (fixed before the kernels first ran).  u = 2^-24 is half a step of fp32.
  The kernels form e = 2^t with t = (x - m) c for a reference m within 2^8 of the row's maximum.  The
  difference, the product and the constant are rounded once each (3 u relative in t) and the
  exponential is good to 2^-22, so a term is off by at most  2^-22 + 3 u ln2 |t|  relative.  Terms
  with |t| > 40 hold less than 2^-40 V of a sum, so |t| <= 40 may be taken: 2.4e-7 + 5.0e-6.  Weighted
  by the terms themselves the mean of |t| is below log2 V + 1.5 <= 19 for any row: 2.4e-7 + 2.4e-6.
  A lane's sum has at most 64 + V / (32 * 64) additions in a chain, one u each, 139 u = 8.3e-6 at
  worst and its square root 0.7e-6 as a rule.  Together LSE = 1.2e-5 absolute on a log-sum-exp or
  a log probability, before they are rounded themselves (u relative).
  Entropy: the same for ln s, and for u / s, whose terms carry a further factor |x - m| / T <= 19 ln2 on
  the mean: ENT = LSE + 13.2 (2.4e-7 + 2.4e-6) + 13.2 * 0.7e-6 = 6e-5.
  Gradient: p is off by 2^-22 + 3 u ln2 |t| with |t| <= 126 (below, p is 0): 1.6e-5, plus the error LSE
  of the log-sum-exp that it is given: 2.8e-5 relative to  p (|a| + |g_H| (|ln p| + H)) ; ENT |g_H| p for
  the entropy that it is given; then one rounding to the output's type.  The exponential gives 0 for
  results below 2^-126, the smallest normal number: p is off by that much at most, which its factor
  |a| + |g_H| (|ln p| + H) multiplies.
"""
import torch

U = 2.0 ** -24
LSE = 1.2e-5
ENT = 6e-5
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def f32(x):
    return float(torch.tensor(float(x), dtype=torch.float32))


def statistics(x, inv_t):
    """x [...,V] any float type, inv_t [...] float64 -> dict of float64 z, p, lp, lse, ent, ok."""
    x = x.double()
    ok = torch.isfinite(x)
    z = torch.where(ok, x * inv_t[..., None], torch.full_like(x, float("-inf")))
    some = ok.any(-1)
    m = torch.where(some, z.amax(-1), torch.zeros_like(inv_t))
    s = torch.exp(z - m[..., None]).sum(-1)
    lse = torch.where(some, m + torch.log(s), torch.full_like(m, float("-inf")))
    lp = torch.where(some[..., None], (z - m[..., None]) - torch.log(s)[..., None], z)
    p = torch.where(some[..., None], torch.exp(lp), torch.zeros_like(lp))
    ent = -torch.where(p > 0, p * lp, torch.zeros_like(p)).sum(-1)
    return dict(z=z, p=p, lp=lp, lse=lse, ent=ent, ok=ok, some=some)


def logprobs(x, tokens, inv_t, M):
    """tokens [...,G] -> dict as token_logprobs returns it, in 64 bits (alternatives exact)."""
    st = statistics(x, inv_t)
    V = x.shape[-1]
    t = tokens.long()
    lp = st["lp"].gather(-1, t.clamp(0, V - 1))
    lp = torch.where(t >= V, torch.full_like(lp, float("-inf")), lp)
    lp = torch.where(t < 0, torch.zeros_like(lp), lp)
    out = dict(logprobs=lp, lse=st["lse"], entropy=st["ent"])
    if M:
        key = torch.where(st["ok"], x.double() + 0.0, torch.full_like(x, float("-inf"), dtype=torch.float64))
        order = key.sort(dim=-1, descending=True, stable=True).indices[..., :M]
        n = st["ok"].sum(-1, keepdim=True)
        ids = torch.full(x.shape[:-1] + (M,), -1, dtype=torch.int64, device=x.device)
        k = min(M, V)
        ids[..., :k] = torch.where(torch.arange(k, device=x.device) < n, order, torch.full_like(order, -1))
        tl = st["lp"].gather(-1, ids.clamp(min=0))
        out["top_ids"] = ids
        out["top_logprobs"] = torch.where(ids < 0, torch.full_like(tl, float("-inf")), tl)
    return out


def near(got, want, tol, what):
    """Infinite results have to be equal, one that rounding to the output's type makes infinite too."""
    stored = want.to(got.dtype).double()
    got, want = got.double(), want.double()
    same = (got == stored) | (torch.isfinite(stored) & ((got - want).abs() <= tol))
    assert bool(same.all()), "%s: %d of %d off, worst %g over tolerance" % (
        what, int((~same).sum()), same.numel(), float(((got - want).abs() - tol)[~same].max()))


def check_logprobs(got, want, what):
    near(got["logprobs"], want["logprobs"], LSE + U * want["logprobs"].abs(), what + " logprobs")
    near(got["lse"], want["lse"], LSE + U * want["lse"].abs(), what + " lse")
    if "entropy" in got:
        near(got["entropy"], want["entropy"], ENT + U * want["entropy"].abs(), what + " entropy")
    if "top_ids" in want:
        assert torch.equal(got["top_ids"].long(), want["top_ids"]), what + " top ids"
        near(got["top_logprobs"], want["top_logprobs"], LSE + U * want["top_logprobs"].abs(), what + " top logprobs")


def gradient(x, tokens, inv_t, g_lp=None, g_lse=None, g_ent=None, top_ids=None, g_top=None):
    """(gradient, its error scale before the last rounding) in 64 bits, by the formula."""
    st = statistics(x, inv_t)
    V = x.shape[-1]
    zero = torch.zeros_like(st["lse"])
    a = zero if g_lse is None else g_lse.double()
    scatter = torch.zeros_like(st["p"])
    for ids, g in ((tokens, g_lp), (top_ids, g_top)):
        if g is None:
            continue
        t = ids.long()
        inside = (t >= 0) & (t < V)
        counts = inside & st["ok"].gather(-1, t.clamp(0, V - 1))
        gg = torch.where(counts, g.double(), torch.zeros_like(g, dtype=torch.float64))
        a = a - gg.sum(-1)
        scatter = scatter.scatter_add(-1, t.clamp(0, V - 1), gg)
    h = zero if g_ent is None else g_ent.double()
    lp = torch.where(st["p"] > 0, st["lp"], torch.zeros_like(st["lp"]))
    d = st["p"] * (a[..., None] - h[..., None] * (lp + st["ent"][..., None])) + scatter
    factor = a.abs()[..., None] + h.abs()[..., None] * (lp.abs() + st["ent"][..., None])
    scale = (st["p"] * 2.8e-5 + 2.0 ** -126) * factor + st["p"] * ENT * h.abs()[..., None] + 4 * U * scatter.abs()
    live = (st["ok"] & st["some"][..., None]).double()
    return d * inv_t[..., None] * live, scale * inv_t[..., None] * live


def check_gradient(got, want, scale, what):
    # 2^-126: results below the smallest normal number may be flushed
    near(got, want, scale + HALF[got.dtype] * want.abs() + 2.0 ** -126 + HALF[got.dtype] * scale, what)
