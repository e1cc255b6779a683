"""Plain 64-bit forms of independent sampling and of 4-bit tables, and the tolerances of their tests.

Tolerances (fixed before the kernels first ran).  u = 2^-24 is half a step of fp32.
  Tokens, codes, scales and zeros are equal: what decides is computed in 64 bits on both sides.
  Log probabilities of a sample are ln w_t - ln total, both in 64 bits unless nothing truncates the row; then the
  total is a sum of fp32 chunk sums whose terms are off by 2^-22 + 3 u |t| (t: the exponent in base 2, |t| <= 9.5 on the
  mean weighted by the terms of a chunk of 256, u relative per rounding) and that a chain of 14 additions
  rounds: 2.4e-7 + 1.7e-6 + 0.8e-6 = 2.8e-6 relative.  SLP = 3e-6 absolute, one more for each doubling of the chunk,
  and u relative for the result's own rounding.
  Logits of a 4-bit head: products of 8-bit by 5-bit integers are exact; an instruction adds 16 of them to its
  accumulator and rounds or cuts to 24 bits, 2 u of what it holds, which S = sum |x w| bounds.  A group of 128 columns
  takes 8 instructions, times three for fp32 x, a step's product and addition two more roundings, and D / 128
  groups or their parts are added up: (2 * 24 + 2 + D / 128 + 16) u S, smaller groups less per group and more groups:
  (2 * 24 + 18 + D / group) u S covers each; then half a step of the output's type.
"""
import torch

U = 2.0 ** -24
SLP = 3e-6
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def f32(x):
    return float(torch.tensor(float(x), dtype=torch.float32))


def sample_row(x, u, inv_temp, top_k, top_p, min_p):
    """x [V] (any float type) and fp32-representable settings -> (token, log probability)."""
    x = x.double() + 0.0
    V = x.numel()
    bad = not (inv_temp > 0) or (inv_temp != float("inf") and not 1e-20 <= inv_temp <= f32(1e20)) or not top_p > 0 \
        or not 0 <= min_p <= 1 or not 0 <= u <= 1
    x = torch.where(torch.isfinite(x), x, torch.full_like(x, float("-inf")))
    if bad or not bool(torch.isfinite(x).any()):
        return -1, 0.0
    if inv_temp == float("inf"):
        return int((x == x.max()).nonzero()[0]), 0.0
    order = x.sort(descending=True, stable=True).indices
    order = order[: int(torch.isfinite(x).sum())]
    z = (x[order] - x[order[0]]) * inv_temp
    w = torch.exp(z)
    n = len(order)
    if 0 < top_k < V:
        n = min(n, top_k)
    if top_p < 1:
        cum = torch.cumsum(w[:n], 0)
        n = max(1, int((cum - w[:n] < top_p * cum[-1]).sum()))
    if min_p > 0:
        n = max(1, min(n, int((z >= torch.log(torch.tensor(min_p, dtype=torch.float64)).to(z.device)).sum())))
    kept = torch.zeros(V, dtype=torch.float64, device=x.device)
    kept[order[:n]] = w[:n]
    cum = torch.cumsum(kept, 0)
    total = cum[-1]
    over = ((cum > u * total) & (kept > 0)).nonzero()
    t = int(over[0]) if len(over) else int((kept > 0).nonzero()[-1])
    return t, float(torch.log(kept[t] / total))


def sample(x, u, inv_temp=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """x [B,K,J,V], u [B,K,J]; settings numbers or tensors that broadcast over [B,K,J] from the left."""
    lead = x.shape[:3]

    def rows(v, dtype):
        v = torch.as_tensor(v, dtype=dtype).cpu()
        return v.reshape(v.shape + (1,) * (3 - v.dim())).expand(lead).reshape(-1).tolist()

    it, k, p, m = rows(inv_temp, torch.float32), rows(top_k, torch.int32), rows(top_p, torch.float32), rows(min_p, torch.float32)
    uu = u.reshape(-1).tolist()
    flat = x.reshape(-1, x.shape[3])
    got = [sample_row(flat[i], uu[i], it[i], k[i], p[i], m[i]) for i in range(flat.shape[0])]
    return torch.tensor([g[0] for g in got]).view(lead), torch.tensor([g[1] for g in got], dtype=torch.float64).view(lead)


def quantize(w, group, zeros, scale_dtype):
    """-> (codes [V,D] 0 .. 15, scales, zeros) in 64 bits with the definition's own roundings."""
    V, D = w.shape
    q, s, z = [], [], []
    for g in range(0, D, group):
        x = w[:, g:g + group].double()
        bad = ~torch.isfinite(x).all(1)
        x = torch.where(bad[:, None], torch.zeros_like(x), x)
        lo, hi = x.amin(1).clamp(max=0.0), x.amax(1).clamp(min=0.0)
        step = ((hi - lo).float().double() / 15.0).float() if zeros else (torch.maximum(-lo, hi) / 7.0).float()
        step = step.to(scale_dtype).double()
        bad |= torch.isinf(step)
        ok = (step > 0) & ~bad
        safe = torch.where(ok, step, torch.ones_like(step))
        zero = (-lo / safe).float().double().round().clamp(0, 15) * ok if zeros else torch.full_like(step, 8.0)
        c = (((x / safe[:, None]).float().double().round()) * ok[:, None] + zero[:, None]).clamp(0, 15)
        c = torch.where(bad[:, None], torch.zeros_like(c), c)
        q.append(c)
        s.append(torch.where(bad, torch.full_like(step, float("nan")), step))
        z.append(torch.where(bad, torch.zeros_like(zero), zero) if zeros else zero)
    return torch.cat(q, 1), torch.stack(s, 1), torch.stack(z, 1)


def unpack(table):
    """(codes [V,dim], zeros [V,G]) of an Int4Table as float64."""
    c = torch.stack([table.codes & 15, table.codes >> 4], -1).flatten(1)[:, :table.dim].double()
    z = torch.full(table.scales.shape, 8.0, dtype=torch.float64, device=c.device) if table.zeros is None \
        else (table.zeros & 15).double()
    return c, z


def rows64(table):
    """The table's elements in 64 bits."""
    c, z = unpack(table)
    g = torch.arange(table.dim, device=c.device) // table.group
    return (c - z[:, g]) * table.scales.double()[:, g]


def rows32(table, scale, dtype):
    """The same as embed_tokens_int4 rounds them."""
    c, z = unpack(table)
    g = torch.arange(table.dim, device=c.device) // table.group
    y = ((c - z[:, g]).float() * table.scales.float()[:, g]) * torch.tensor(scale, dtype=torch.float32, device=c.device)
    return y.to(dtype)


def check_logits(got, x, table, what=""):
    w = rows64(table)
    want = x.double().reshape(-1, table.dim) @ w.T
    mass = x.double().abs().reshape(-1, table.dim) @ w.abs().T
    tol = (66 + table.dim / table.group) * U * mass + HALF[got.dtype] * want.abs() * (1 + 1e-3) + 1e-37
    off = (got.double().reshape(want.shape) - want).abs()
    assert bool((off <= tol).all()), "%s: worst %g of its tolerance" % (what, float((off / tol).nan_to_num(1e9).max()))
