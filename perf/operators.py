"""Cases and plain forms of the operators at the two vocabulary-sized ends of a drafter: the log
probabilities of given tokens (with entropy and top alternatives) and their gradient, and the
embedding lookup of tokens and its gradient.

A case's "op" is one of

    logprobs     rows of logits [B,K,J,V], one token per row -> log probability, log-sum-exp,
                 entropy, the M most likely tokens and their log probabilities
    emitted      the same for the tokens a verification emitted: one row per emitted position
    grad         gradient of log probabilities (and entropies) with respect to the logits
    embed        rows of a table [V,D] by token, scaled; token -1 gives zeros
    embed_grad   gradient of that with respect to the table
"""
import math

import torch

own = False

_DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "bf16": 2}


def listed():
    return [
        # one position of one sequence: what a chat front end asks after every token it shows
        dict(name="logprobs_one_row", op="logprobs", B=1, K=1, J=1, V=152064, dtype="bf16", M=20,
             inv_temp=1.0, masked=128),
        # the drafts of a small fp32 step (8 sequences, 4 drafts, 4 positions)
        dict(name="logprobs_small_fp32", op="logprobs", B=8, K=4, J=4, V=32000, dtype="f32", M=8,
             inv_temp=1.25, masked=0),
        # scoring a large batch of drafts: 8192 rows, 2.5 GB
        dict(name="logprobs_large", op="logprobs", B=128, K=8, J=8, V=152064, dtype="bf16", M=20,
             inv_temp=1.0, masked=128),
        # the answer of a serving step: the tokens that a verification of 8 drafts of 5 emitted
        dict(name="emitted_serving", op="emitted", B=64, K=8, J=6, V=128256, dtype="bf16", M=5,
             inv_temp=1.25, masked=0),
        # training the drafter on one small fp32 batch
        dict(name="grad_small_fp32", op="grad", B=8, K=4, J=4, V=32000, dtype="f32", inv_temp=1.0,
             masked=0, entropy=True),
        # a vocabulary whose rows start on no boundary, with an entropy bonus
        dict(name="grad_odd_vocabulary", op="grad", B=32, K=4, J=5, V=50257, dtype="bf16",
             inv_temp=1.25, masked=0, entropy=True),
        # training on a large batch: 4096 rows, 1.25 GB read and written
        dict(name="grad_large", op="grad", B=64, K=8, J=8, V=152064, dtype="bf16", inv_temp=1.0,
             masked=128, entropy=False),
        # the inputs of the next draft position: 64 sequences, 8 drafts
        dict(name="embed_decode", op="embed", N=512, V=128256, D=4096, dtype="bf16", scale=1.0,
             padded=0.0),
        # prompts and training batches
        dict(name="embed_prefill", op="embed", N=65536, V=128256, D=4096, dtype="bf16", scale=64.0,
             padded=0.02),
        # candidates chosen by the decoders of the compression scheme: 16 fp32 coordinates each
        dict(name="embed_candidates", op="embed", N=2048, V=1048576, D=16, dtype="f32", scale=0.75,
             padded=0.01),
        # training a small drafter on a short batch
        dict(name="embed_grad_small_fp32", op="embed_grad", N=2048, V=32000, D=1024, dtype="f32",
             scale=32.0, padded=0.02),
        # training a larger one on a long batch
        dict(name="embed_grad_large", op="embed_grad", N=65536, V=128256, D=4096, dtype="bf16",
             scale=1.0, padded=0.02),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["logprobs", "emitted", "grad", "embed", "embed_grad"])
    dtype = rng.choice(["f32", "bf16", "bf16"])
    if op in ("logprobs", "emitted", "grad"):
        K, J = rng.randint(1, 8), rng.randint(2 if op == "emitted" else 1, 9)
        V = _log_int(rng, 1000, 152064)
        most = {"logprobs": 8192, "emitted": 4096, "grad": 4096}[op] * 152064 * 2 // _BYTES[dtype]
        B = _log_int(rng, 1, max(1, min(512, most // (K * J * V))))
        c = dict(op=op, B=B, K=K, J=J, V=V, dtype=dtype, inv_temp=rng.choice([0.5, 1.0, 1.25, 2.0]),
                 masked=rng.choice([0, 0, 1, 128]))
        if op == "grad":
            c["entropy"] = rng.random() < 0.5
        else:
            c["M"] = rng.choice([0, 1, 5, 20, 33, 50])
        return c
    V = _log_int(rng, 1000, 1048576)
    D = min(_log_int(rng, 16, 8192), (1 << 29) // V)
    N = min(_log_int(rng, 1, 131072), (1 << 28) // D)
    return dict(op=op, N=N, V=V, D=D, dtype=dtype, scale=rng.choice([1.0, 0.75, 45.25]),
                padded=rng.choice([0.0, 0.02, 0.3]))


def _logits(c, gen):
    """Normal logits of standard deviation 4 with one token in a hundred 8 higher; the last
    `masked` tokens of the vocabulary are padding and can not be drawn (-inf)."""
    B, K, J, V = c["B"], c["K"], c["J"], c["V"]
    x = torch.empty((B * K * J, V), dtype=_DTYPES[c["dtype"]], device="cuda")
    step = max(1, (1 << 27) // V)
    for r in range(0, x.shape[0], step):
        n = min(step, x.shape[0] - r)
        y = 4.0 * torch.randn((n, V), generator=gen, device="cuda")
        y += 8.0 * (torch.rand((n, V), generator=gen, device="cuda") < 0.01)
        x[r:r + n] = y.to(x.dtype)
    if c["masked"]:
        x[:, V - c["masked"]:] = float("-inf")
    return x.view(B, K, J, V)


def _sampled(rows, inv_temp, gen):
    """One token per row [R,V], drawn from softmax(rows * inv_temp)."""
    out = torch.empty(rows.shape[0], dtype=torch.int32, device="cuda")
    step = max(1, (1 << 27) // rows.shape[1])
    for r in range(0, rows.shape[0], step):
        x = rows[r:r + step].float() * inv_temp
        e = torch.empty_like(x).exponential_(generator=gen)
        out[r:r + step] = (x - e.log()).argmax(-1).to(torch.int32)
    return out


def _emitted_rows(accept, B, K, J):
    """The draft whose row an emitted position is drawn from: the lowest one still active."""
    active = torch.cat([torch.ones((B, K, 1), dtype=torch.uint8, device="cuda"), accept], 2)
    return (active != 0).to(torch.uint8).argmax(1)  # [B,J]; 0 where none is active


def _statistics64(x, inv_temp):
    """Log-sum-exp and entropy of each row of x [R,V], in 64 bits."""
    lse = torch.empty(x.shape[0], dtype=torch.float64, device="cuda")
    ent = torch.empty_like(lse)
    step = max(1, (1 << 26) // x.shape[1])
    for r in range(0, x.shape[0], step):
        z = x[r:r + step].double() * inv_temp
        l1 = torch.logsumexp(z, -1, keepdim=True)
        lp = z - l1
        p = lp.exp()
        lse[r:r + step] = l1[:, 0]
        ent[r:r + step] = -torch.where(p > 0, p * lp, torch.zeros_like(p)).sum(-1)
    return lse, ent


def prepare(case, seed):
    c = dict(case)
    gen = torch.Generator(device="cuda").manual_seed(seed * 1000003 + 17)
    op = c["op"]
    s = dict(c=c)
    if op in ("logprobs", "emitted", "grad"):
        B, K, J, V = c["B"], c["K"], c["J"], c["V"]
        s["logits"] = _logits(c, gen)
        flat = s["logits"].view(-1, V)
        if op == "emitted":
            L = J - 1
            # sequence lengths 1 .. J in equal numbers, in a random order; one draft carries each
            tau = (1 + torch.arange(B, device="cuda") % J)[torch.randperm(B, generator=gen, device="cuda")]
            reach = (torch.rand((B, K), generator=gen, device="cuda") * tau[:, None]).long()
            carrier = torch.randint(K, (B,), generator=gen, device="cuda")
            reach[torch.arange(B, device="cuda"), carrier] = tau - 1
            s["accept"] = (torch.arange(L, device="cuda") < reach[:, :, None]).to(torch.uint8)
            k = _emitted_rows(s["accept"], B, K, J)
            j = torch.arange(J, device="cuda").expand(B, J)
            row = (torch.arange(B, device="cuda")[:, None] * K + k) * J + j
            tok = _sampled(flat[row.reshape(-1)], c["inv_temp"], gen).view(B, J)
            s["tokens"] = torch.where(j < tau[:, None], tok, torch.full_like(tok, -1)).contiguous()
            return s
        s["tokens"] = _sampled(flat, c["inv_temp"], gen).view(B, K, J)
        if op == "grad":
            lse, ent = _statistics64(flat, c["inv_temp"])
            s["lse"], s["ent"] = lse.float().view(B, K, J), ent.float().view(B, K, J)
            s["g_lp"] = torch.randn((B, K, J), generator=gen, device="cuda")
            s["g_ent"] = 0.1 * torch.randn((B, K, J), generator=gen, device="cuda") if c["entropy"] else None
        return s
    N, V, D = c["N"], c["V"], c["D"]
    # token frequencies fall off as 1 / rank; a share of the positions is padding
    rank = torch.exp(torch.rand(N, generator=gen, device="cuda", dtype=torch.float64) * math.log(V)).long().clamp_(1, V) - 1
    tok = (rank * 7919 + 13) % V
    tok = torch.where(torch.rand(N, generator=gen, device="cuda") < c["padded"], torch.full_like(tok, -1), tok)
    s["tokens"] = tok.to(torch.int32)
    x = torch.empty((V if op == "embed" else N, D), dtype=_DTYPES[c["dtype"]], device="cuda")
    step = max(1, (1 << 27) // D)
    for r in range(0, x.shape[0], step):
        n = min(step, x.shape[0] - r)
        x[r:r + n] = torch.randn((n, D), generator=gen, device="cuda").to(x.dtype)
    s["x"] = x
    return s


def _plain_logprobs(x, tok, inv_temp, M):
    """x [R,V], tok [R] (>= 0)."""
    z = x.float() * inv_temp
    m = z.amax(-1, keepdim=True)
    e = torch.exp(z - m)
    total = e.sum(-1, keepdim=True)
    lse = m + torch.log(total)
    d = torch.where(e > 0, z - m, torch.zeros_like(z))
    ent = torch.log(total) - (e * d).sum(-1, keepdim=True) / total
    out = dict(logprobs=(z.gather(1, tok.long()[:, None]) - lse)[:, 0], lse=lse[:, 0], entropy=ent[:, 0])
    if M:
        # one integer per logit that orders by value, then by lower index
        bits = (x.float() + 0.0).view(torch.int32)
        order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long()
        key = (order << 32) | (0x7FFFFFFF - torch.arange(x.shape[1], device=x.device))
        ids = 0x7FFFFFFF - (key.topk(M, -1).values & 0xFFFFFFFF)
        out["top_ids"] = ids.to(torch.int32)
        out["top_logprobs"] = z.gather(1, ids) - lse
    return out


def run(state):
    c = state["c"]
    op = c["op"]
    if own:
        import paper_2506_05632_b200 as gls

        if op == "logprobs":
            return gls.token_logprobs(state["logits"], state["tokens"], top=c["M"], inv_temp=c["inv_temp"])
        if op == "emitted":
            return gls.emitted_logprobs(state["logits"], state["tokens"], state["accept"], top=c["M"],
                                        inv_temp=c["inv_temp"])
        if op == "grad":
            return gls.token_logprobs_backward(state["logits"], state["tokens"], state["lse"],
                                               entropy=state["ent"], grad_logprobs=state["g_lp"],
                                               grad_entropy=state["g_ent"], inv_temp=c["inv_temp"])
        if op == "embed":
            return gls.embed_tokens(state["x"], state["tokens"], scale=c["scale"])
        return gls.embed_tokens_backward(state["x"], state["tokens"], c["V"], scale=c["scale"])
    if op in ("logprobs", "emitted", "grad"):
        B, K, J, V = c["B"], c["K"], c["J"], c["V"]
        if op == "logprobs":
            o = _plain_logprobs(state["logits"].view(-1, V), state["tokens"].view(-1), c["inv_temp"], c["M"])
            return {k: v.reshape((B, K, J) + v.shape[1:]) for k, v in o.items()}
        if op == "emitted":
            k = _emitted_rows(state["accept"], B, K, J)
            b = torch.arange(B, device="cuda")[:, None]
            x = state["logits"][b, k, torch.arange(J, device="cuda")].view(-1, V)
            o = _plain_logprobs(x, state["tokens"].view(-1).clamp(min=0), c["inv_temp"], c["M"])
            live = state["tokens"].view(-1) >= 0
            for name, v in list(o.items()):
                keep = live if v.dim() == 1 else live[:, None]
                v = torch.where(keep, v, torch.full_like(v, -1 if name == "top_ids" else 0))
                o[name] = v.reshape((B, J) + v.shape[1:])
            return o
        lp = state["logits"].float() * c["inv_temp"] - state["lse"][..., None]
        p = torch.exp(lp)
        weight = -state["g_lp"][..., None]
        if state["g_ent"] is not None:
            lp = torch.where(p > 0, lp, torch.zeros_like(lp))
            weight = weight - state["g_ent"][..., None] * (lp + state["ent"][..., None])
        d = p * weight
        d.scatter_add_(3, state["tokens"].long()[..., None], state["g_lp"][..., None])
        return (d * c["inv_temp"]).to(state["logits"].dtype)
    tok = state["tokens"].long()
    live = (tok >= 0)[:, None]
    if op == "embed":
        rows = state["x"][tok.clamp(min=0)].float() * c["scale"]
        return torch.where(live, rows, torch.zeros_like(rows)).to(state["x"].dtype)
    g = torch.where(live, state["x"].float(), torch.zeros((), device="cuda"))
    d = torch.zeros((c["V"], c["D"]), device="cuda").index_add_(0, tok.clamp(min=0), g)
    return (d * c["scale"]).to(state["x"].dtype)


def work(case):
    c = case
    es = _BYTES[c["dtype"]]
    op = c["op"]
    if op in ("logprobs", "emitted", "grad"):
        rows = c["B"] * c["K"] * c["J"]
        if op == "emitted":
            rows = sum(1 + b % c["J"] for b in range(c["B"]))
        n = rows * c["V"]
        if op == "grad":
            return dict(bytes=2 * n * es + rows * 20, flops=6 * n)
        return dict(bytes=n * es + rows * (16 + 8 * c["M"]), flops=6 * n)
    N, V, D = c["N"], c["V"], c["D"]
    kept = int(N * (1 - c["padded"]))
    if op == "embed":
        return dict(bytes=4 * N + (kept + N) * D * es, flops=N * D)
    return dict(bytes=4 * N + (kept + V) * D * es, flops=kept * D)


def exact(case, seed):
    s = prepare(case, seed)
    c = s["c"]
    op = c["op"]
    if op in ("logprobs", "emitted"):
        B, K, J, V, M = c["B"], c["K"], c["J"], c["V"], c["M"]
        if op == "logprobs":
            lead, rows = (B, K, J), s["logits"].view(-1, V)
        else:
            lead = (B, J)
            k = _emitted_rows(s["accept"], B, K, J)
            at = (torch.arange(B, device="cuda")[:, None] * K + k) * J + torch.arange(J, device="cuda")
            rows = s["logits"].view(-1, V)[at.view(-1)]
        tok = s["tokens"].reshape(-1).long()
        lse, ent = _statistics64(rows, c["inv_temp"])
        out = dict(logprobs=rows.gather(1, tok.clamp(min=0)[:, None])[:, 0].double() * c["inv_temp"] - lse,
                   lse=lse, entropy=ent)
        if M:
            # stable ordering by value keeps the lower index first
            ids = torch.empty((rows.shape[0], M), dtype=torch.int64, device="cuda")
            step = max(1, (1 << 26) // V)
            for r in range(0, rows.shape[0], step):
                ids[r:r + step] = rows[r:r + step].float().sort(dim=-1, descending=True, stable=True).indices[:, :M]
            out["top_ids"] = ids
            out["top_logprobs"] = rows.gather(1, ids).double() * c["inv_temp"] - lse[:, None]
        for name, v in list(out.items()):
            gone = (tok < 0) if v.dim() == 1 else (tok < 0)[:, None]
            out[name] = v.masked_fill(gone, -1 if name == "top_ids" else 0).reshape(lead + v.shape[1:])
        return out
    if op == "grad":
        V = c["V"]
        x = s["logits"].view(-1, V)
        tok, g = s["tokens"].view(-1).long(), s["g_lp"].view(-1).double()
        h = None if s["g_ent"] is None else s["g_ent"].view(-1).double()
        out = torch.empty(x.shape, dtype=torch.float64, device="cuda")
        lse, ent = _statistics64(x, c["inv_temp"])
        step = max(1, (1 << 26) // V)
        for r in range(0, x.shape[0], step):
            lp = x[r:r + step].double() * c["inv_temp"] - lse[r:r + step, None]
            p = lp.exp()
            one = torch.zeros_like(p)
            one[torch.arange(p.shape[0], device="cuda"), tok[r:r + step]] = 1.0
            d = (one - p) * g[r:r + step, None]
            if h is not None:
                lp = lp.masked_fill(p == 0, 0.0)
                d -= p * (lp + ent[r:r + step, None]) * h[r:r + step, None]
            out[r:r + step] = d * c["inv_temp"]
        return out.view(s["logits"].shape)
    tok = s["tokens"].long()
    if op == "embed":
        rows = s["x"][tok.clamp(min=0)].double() * c["scale"]
        rows[tok < 0] = 0.0
        return rows
    d = torch.zeros((c["V"], c["D"]), dtype=torch.float64, device="cuda")
    some = tok >= 0
    d.index_add_(0, tok[some], s["x"][some].double())
    return d * c["scale"]
