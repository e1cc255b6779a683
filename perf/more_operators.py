"""Cases and plain forms of a drafter's vocabulary-sized ends on 4-bit weights and of independent
sampling between them: the logits of hidden states from a 4-bit head, a token per row of logits by
temperature, top-k, top-p and min-p from a given uniform number, and the 4-bit table itself, made from
weights and read back by token.

A case's "op" is one of

    sample   rows of logits [B,K,J,V] and a uniform number per row -> tokens and their log
             probabilities under the truncated distribution.  A row's order is by logit, ties by
             lower index; top-k keeps the first k, top-p the shortest start of those that holds
             top_p of their mass, min-p what is at least min_p times as likely as the first.  The
             token is the first by index whose cumulative mass among the kept exceeds u times their
             total.  An infinite inverse temperature takes the first token of the order.
    head     x [N,D] times the rows of a 4-bit table of V rows -> logits [N,V].  The element (v, d)
             stands for scale[v, d / group] * (code - zero[v, d / group]), zero 8 where there are none
    table    weights [V,D] -> codes, scales and zeros, and the rows of all tokens read back
"""
import math

import torch

own = False

_DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "bf16": 2}


def listed():
    return [
        # the next token of one conversation
        dict(name="sample_one_row", op="sample", B=1, K=1, J=1, V=152064, dtype="bf16", masked=128,
             inv_temp=1.25, top_k=50, top_p=0.9, min_p=0.0, requests=False),
        # the drafts of a small fp32 step by nucleus sampling
        dict(name="sample_small_fp32", op="sample", B=8, K=4, J=1, V=32000, dtype="f32", masked=0,
             inv_temp=1.0, top_k=0, top_p=0.95, min_p=0.0, requests=False),
        # a vocabulary whose rows start on no boundary
        dict(name="sample_odd_vocabulary", op="sample", B=32, K=4, J=5, V=50257, dtype="bf16", masked=0,
             inv_temp=1.0, top_k=0, top_p=1.0, min_p=0.05, requests=False),
        # a serving batch in which every sequence has settings of its own, greedy ones among them
        dict(name="sample_requests", op="sample", B=64, K=8, J=1, V=128256, dtype="bf16", masked=0,
             inv_temp=1.0, top_k=0, top_p=1.0, min_p=0.0, requests=True),
        # independent drafts of a large batch, a plain draw by temperature: 2048 rows, 0.6 GB
        dict(name="sample_large", op="sample", B=64, K=8, J=4, V=152064, dtype="bf16", masked=128,
             inv_temp=1.0, top_k=0, top_p=1.0, min_p=0.0, requests=False),
        # one position of a small fp32 drafter, latency
        dict(name="head_small_fp32", op="head", N=1, V=32000, D=1024, dtype="f32", out="f32", group=32,
             zeros=False, scales="f32"),
        # one token through a large head
        dict(name="head_one_row", op="head", N=1, V=152064, D=4096, dtype="bf16", out="f32", group=128,
             zeros=True, scales="bf16"),
        # the eight drafts of one sequence
        dict(name="head_drafts", op="head", N=8, V=128256, D=4096, dtype="bf16", out="bf16", group=64,
             zeros=False, scales="bf16"),
        # a vocabulary and a width that fill no tile, three sequences
        dict(name="head_odd", op="head", N=3, V=50257, D=1000, dtype="bf16", out="bf16", group=32,
             zeros=True, scales="f32"),
        # eight drafts of eight sequences
        dict(name="head_batch", op="head", N=64, V=152064, D=4096, dtype="bf16", out="bf16", group=128,
             zeros=True, scales="bf16"),
        # a small fp32 table
        dict(name="table_small_fp32", op="table", V=32000, D=1024, dtype="f32", group=32, zeros=False,
             scales="f32"),
        # a large one
        dict(name="table_large", op="table", V=128256, D=4096, dtype="bf16", group=64, zeros=True,
             scales="bf16"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["sample", "sample", "head", "head", "table"])
    dtype = rng.choice(["f32", "bf16", "bf16"])
    V = _log_int(rng, 1000, 152064)
    if op == "sample":
        K, J = rng.randint(1, 8), rng.randint(1, 4)
        B = _log_int(rng, 1, max(1, min(256, 2048 * 152064 * 2 // _BYTES[dtype] // (K * J * V))))
        return dict(op=op, B=B, K=K, J=J, V=V, dtype=dtype, masked=rng.choice([0, 0, 1, 128]),
                    inv_temp=rng.choice([0.5, 0.8, 1.0, 1.25, 2.0]), top_k=rng.choice([0, 0, 1, 20, 50, 400, 5000]),
                    top_p=rng.choice([1.0, 1.0, 0.8, 0.9, 0.95, 0.99]), min_p=rng.choice([0.0, 0.0, 0.0, 0.02, 0.1]),
                    requests=rng.random() < 0.25)
    D = _log_int(rng, 64, 8192)
    V = max(64, min(V, 152064 * 4096 // D))
    c = dict(op=op, V=V, D=D, dtype=dtype, group=rng.choice([32, 64, 128]), zeros=rng.random() < 0.5,
             scales=rng.choice(["f32", "bf16"]))
    if op == "table":
        c["V"] = max(64, min(V, 128256 * 4096 * 2 // _BYTES[dtype] // D))
        return c
    c["N"] = _log_int(rng, 1, 64)
    c["out"] = rng.choice(["f32", dtype])
    return c


def _logits(c, gen):
    """Normal logits of standard deviation 4 with one token in a hundred 8 higher, times a factor per row
    that makes some rows peaked and others flat; the last `masked` tokens are padding (-inf)."""
    B, K, J, V = c["B"], c["K"], c["J"], c["V"]
    R = B * K * J
    x = torch.empty((R, V), dtype=_DTYPES[c["dtype"]], device="cuda")
    sharp = torch.exp(torch.rand((R, 1), generator=gen, device="cuda") * math.log(2.0) + math.log(0.75))
    step = max(1, (1 << 27) // V)
    for r in range(0, R, step):
        n = min(step, R - r)
        y = 4.0 * torch.randn((n, V), generator=gen, device="cuda")
        y += 8.0 * (torch.rand((n, V), generator=gen, device="cuda") < 0.01)
        x[r:r + n] = (y * sharp[r:r + n]).to(x.dtype)
    if c["masked"]:
        x[:, V - c["masked"]:] = float("-inf")
    return x.view(B, K, J, V)


def _choice(values, n, dtype, gen):
    v = torch.tensor(values, dtype=dtype, device="cuda")
    return v[torch.randint(len(values), (n,), generator=gen, device="cuda")]


def prepare(case, seed):
    c = dict(case)
    gen = torch.Generator(device="cuda").manual_seed(seed * 1000003 + 29)
    s = dict(c=c)
    if c["op"] == "sample":
        B, K, J = c["B"], c["K"], c["J"]
        s["logits"] = _logits(c, gen)
        s["u"] = torch.rand((B, K, J), generator=gen, device="cuda")
        s["set"] = {n: c[n] for n in ("inv_temp", "top_k", "top_p", "min_p")}
        if c["requests"]:  # one setting per sequence
            s["set"] = dict(inv_temp=_choice([0.8, 1.0, 1.0, 1.25, 2.0, math.inf], B, torch.float32, gen),
                            top_k=_choice([0, 0, 20, 50, 1000], B, torch.int32, gen),
                            top_p=_choice([1.0, 1.0, 0.9, 0.95], B, torch.float32, gen),
                            min_p=_choice([0.0, 0.0, 0.0, 0.05], B, torch.float32, gen))
        return s
    V, D = c["V"], c["D"]
    if c["op"] == "table":
        s["w"] = torch.empty((V, D), dtype=_DTYPES[c["dtype"]], device="cuda")
        step = max(1, (1 << 27) // D)
        for r in range(0, V, step):
            n = min(step, V - r)
            s["w"][r:r + n] = (0.02 * torch.randn((n, D), generator=gen, device="cuda")).to(s["w"].dtype)
        s["all"] = torch.arange(V, dtype=torch.int32, device="cuda")
        return s
    # a table as a program holds it: two codes a byte, the even column in the low half, rows on 16-byte boundaries
    G, pitch = -(-D // c["group"]), -(-D // 32) * 16
    s["codes"] = torch.empty((V, pitch), dtype=torch.uint8, device="cuda")
    step = max(1, (1 << 26) // pitch)
    for r in range(0, V, step):
        n = min(step, V - r)
        q = (8.0 + 2.7 * torch.randn((n, pitch, 2), generator=gen, device="cuda")).round_().clamp_(0, 15).to(torch.uint8)
        s["codes"][r:r + n] = q[..., 0] | q[..., 1] << 4
    s["scales"] = (0.015 + 0.01 * torch.rand((V, G), generator=gen, device="cuda")).to(_DTYPES[c["scales"]])
    s["zeros"] = torch.randint(6, 11, (V, G), generator=gen, device="cuda", dtype=torch.uint8) if c["zeros"] else None
    s["x"] = torch.randn((c["N"], D), generator=gen, device="cuda").to(_DTYPES[c["dtype"]])
    return s


def _plain_sample(x, u, it, top_k, top_p, min_p):
    """x [R,V] in fp32 with -inf where masked; u and the settings [R,1] in 64 bits."""
    V = x.shape[1]
    order = (x + 0.0).sort(dim=-1, descending=True, stable=True)
    z = order.values.double()
    z = z - z[:, :1]
    greedy = torch.isinf(it)
    z = z * torch.where(greedy, torch.ones_like(it), it)
    w = torch.exp(z)
    rank = torch.arange(V, device=x.device)
    keep = (rank < torch.where(greedy, torch.ones_like(top_k), top_k)) & (w > 0)
    cum = torch.cumsum(w * keep, -1)
    keep &= (cum - w < top_p * cum[:, -1:]) | (top_p >= 1)
    keep &= (z >= torch.log(min_p)) | (min_p <= 0)
    keep[:, 0] = True
    w = w * keep
    by_index = torch.zeros_like(w).scatter_(1, order.indices, w)
    cum = torch.cumsum(by_index, -1)
    total = cum[:, -1:]
    token = ((cum > u * total) & (by_index > 0)).to(torch.uint8).argmax(-1, keepdim=True)
    return token[:, 0].to(torch.int32), torch.log(by_index.gather(1, token) / total)[:, 0].float()


def _settings(s, V):
    """(u, inverse temperature, top-k, top-p, min-p), each [R,1] in 64 bits as the fp32 numbers they are."""
    B, K, J = s["u"].shape
    out = [s["u"].double().view(-1, 1)]
    for name, t in (("inv_temp", torch.float32), ("top_k", torch.int32), ("top_p", torch.float32), ("min_p", torch.float32)):
        v = torch.as_tensor(s["set"][name], dtype=t, device="cuda").double()
        v = v.view(-1, 1, 1).expand(B, K, J).reshape(-1, 1)
        out.append(torch.where((v <= 0) | (v > V), torch.full_like(v, V), v) if name == "top_k" else v)
    return out


def _plain_rows(codes, scales, zeros, D, group):
    """fp32 rows of a 4-bit table."""
    q = torch.stack([codes & 15, codes >> 4], -1).view(codes.shape[0], -1)[:, :D].float()
    g = torch.arange(D, device=codes.device) // group
    return (q - (8.0 if zeros is None else zeros.float()[:, g])) * scales.float()[:, g]


def _plain_table(w, group, zeros, scale_dtype):
    """Codes, scales and zeros of fp32 weights [V,D]: one step per group, its zero among the codes."""
    V, D = w.shape
    G = -(-D // group)
    x = torch.zeros((V, G * group), device=w.device)
    x[:, :D] = w
    x = x.view(V, G, group)
    if zeros:
        lo, hi = x.amin(-1).clamp(max=0), x.amax(-1).clamp(min=0)
        scale = ((hi - lo) / torch.full_like(hi, 15.0)).to(scale_dtype)
        step = scale.float()
        zero = torch.where(step > 0, (-lo / step).round().clamp(0, 15), torch.zeros_like(step))
    else:
        top = x.abs().amax(-1)
        scale = (top / torch.full_like(top, 7.0)).to(scale_dtype)
        step = scale.float()
        zero = torch.full_like(step, 8.0)
    q = torch.where(step[..., None] > 0, x / step[..., None], torch.zeros_like(x)).round() + zero[..., None]
    return q.clamp(0, 15).view(V, G * group)[:, :D], scale, zero


def run(state):
    s, c = state, state["c"]
    op = c["op"]
    if own:
        import paper_2506_05632_b200 as gls

        if op == "sample":
            return gls.sample_tokens(s["logits"], s["u"], **s["set"])
        if op == "head":
            table = gls.Int4Table(s["codes"], s["scales"], s["zeros"], c["D"], c["group"])
            return gls.head_logits(s["x"], table, dtype=_DTYPES[c["out"]])
        table = gls.quantize_table(s["w"], group=c["group"], zeros=c["zeros"], scale_dtype=_DTYPES[c["scales"]])
        return dict(scales=table.scales, zeros=table.zeros,
                    values=gls.embed_tokens_int4(table, s["all"], dtype=_DTYPES[c["dtype"]]))
    if op == "sample":
        B, K, J, V = c["B"], c["K"], c["J"], c["V"]
        x = s["logits"].view(-1, V)
        settings = _settings(s, V)
        tokens = torch.empty(x.shape[0], dtype=torch.int32, device="cuda")
        lp = torch.empty(x.shape[0], device="cuda")
        step = max(1, (1 << 27) // V)
        for r in range(0, x.shape[0], step):
            tokens[r:r + step], lp[r:r + step] = _plain_sample(x[r:r + step].float(), *[v[r:r + step] for v in settings])
        return dict(tokens=tokens.view(B, K, J), logprobs=lp.view(B, K, J))
    V, D, group = c["V"], c["D"], c["group"]
    step = max(1, (1 << 27) // D)
    if op == "head":
        x = s["x"].float()
        out = torch.empty((c["N"], V), dtype=_DTYPES[c["out"]], device="cuda")
        for v in range(0, V, step):
            zeros = None if s["zeros"] is None else s["zeros"][v:v + step]
            out[:, v:v + step] = x @ _plain_rows(s["codes"][v:v + step], s["scales"][v:v + step], zeros, D, group).T
        return out
    G = -(-D // group)
    scales = torch.empty((V, G), dtype=_DTYPES[c["scales"]], device="cuda")
    zeros = torch.empty((V, G), dtype=torch.uint8, device="cuda") if c["zeros"] else None
    values = torch.empty((V, D), dtype=_DTYPES[c["dtype"]], device="cuda")
    for v in range(0, V, step):
        q, scale, zero = _plain_table(s["w"][v:v + step].float(), group, c["zeros"], scales.dtype)
        scales[v:v + step] = scale
        if zeros is not None:
            zeros[v:v + step] = zero.to(torch.uint8)
        g = torch.arange(D, device="cuda") // group
        values[v:v + step] = ((q - zero[:, g]) * scale.float()[:, g]).to(values.dtype)
    return dict(scales=scales, zeros=zeros, values=values)


def work(case):
    c = case
    if c["op"] == "sample":
        rows = c["B"] * c["K"] * c["J"]
        return dict(bytes=rows * (c["V"] * _BYTES[c["dtype"]] + 12), flops=2 * rows * c["V"])
    V, D = c["V"], c["D"]
    table = V * ((D + 1) // 2 + -(-D // c["group"]) * (_BYTES[c["scales"]] + (1 if c["zeros"] else 0)))
    if c["op"] == "head":
        return dict(bytes=table + c["N"] * (D * _BYTES[c["dtype"]] + V * _BYTES[c["out"]]), flops=2 * c["N"] * V * D)
    return dict(bytes=2 * table + 2 * V * D * _BYTES[c["dtype"]], flops=6 * V * D)


def exact(case, seed):
    s = prepare(case, seed)
    c = s["c"]
    if c["op"] == "sample":
        V = c["V"]
        rows = s["logits"].view(-1, V)
        settings = _settings(s, V)
        tokens = torch.empty(rows.shape[0], dtype=torch.int64, device="cuda")
        lp = torch.empty(rows.shape[0], dtype=torch.float64, device="cuda")
        step = max(1, (1 << 26) // V)
        at = torch.arange(V, device="cuda")
        for r in range(0, rows.shape[0], step):
            x = rows[r:r + step].double()
            u, it, k, p, m = [v[r:r + step] for v in settings]
            first = x.argmax(-1)  # of equal ones any; the greedy rows look for the lowest below
            top = x.gather(1, first[:, None])
            greedy = torch.isinf(it)
            e = ((x - top) * it.masked_fill(greedy, 1.0)).exp()
            # position of each token in the row's order
            back = x.flip(-1).argsort(dim=-1, stable=True).flip(-1)
            place = torch.empty_like(back).scatter_(1, V - 1 - back, at.expand_as(back).contiguous())
            kept = place < k
            # mass in front of each token of the order, of those that top-k keeps
            sorted_e = (e * kept).gather(1, V - 1 - back)
            front = sorted_e.cumsum(-1) - sorted_e
            inside = front < p * sorted_e.sum(-1, keepdim=True)
            kept &= inside.gather(1, place) | (p >= 1)
            kept &= ((x - top) * it >= m.log()) | (m <= 0)
            kept |= place == 0
            kept &= ~greedy | (place == 0)
            e = e * kept
            total = e.sum(-1)
            reached = e.cumsum(-1) > u * total[:, None]
            token = torch.where(reached & (e > 0), at, V).amin(-1)
            tokens[r:r + step] = token
            lp[r:r + step] = e.gather(1, token[:, None])[:, 0].log() - total.log()
        lead = s["u"].shape
        return dict(tokens=tokens.view(lead), logprobs=lp.view(lead))
    V, D, group = c["V"], c["D"], c["group"]
    if c["op"] == "head":
        x = s["x"].double()
        out = torch.empty((c["N"], V), dtype=torch.float64, device="cuda")
        step = max(1, (1 << 26) // D)
        for v in range(0, V, step):
            byte = s["codes"][v:v + step].long()
            w = torch.empty((byte.shape[0], 2 * byte.shape[1]), dtype=torch.float64, device="cuda")
            w[:, 0::2] = (byte % 16).double()
            w[:, 1::2] = (byte // 16).double()
            zero = 8.0 if s["zeros"] is None else s["zeros"][v:v + step].double().repeat_interleave(group, 1)[:, :D]
            w = (w[:, :D] - zero) * s["scales"][v:v + step].double().repeat_interleave(group, 1)[:, :D]
            out[:, v:v + step] = torch.einsum("nd,vd->nv", x, w)
        return out
    # the definition's own roundings: the step to fp32 and to its type, the quotient to fp32
    scales, zeros = [], []
    values = torch.empty((V, D), dtype=torch.float64, device="cuda")
    for g0 in range(0, D, group):
        w = s["w"][:, g0:g0 + group].double()
        if c["zeros"]:
            low, high = w.amin(1).clamp(max=0.0), w.amax(1).clamp(min=0.0)
            step = ((high - low).float().double() / 15.0).float().to(_DTYPES[c["scales"]])
            some = step > 0
            zero = torch.where(some, (-low / step.double()).float().double().round().clamp(0.0, 15.0), 0.0)
        else:
            step = (w.abs().amax(1) / 7.0).float().to(_DTYPES[c["scales"]])
            some = step > 0
            zero = torch.full_like(step, 8.0, dtype=torch.float64)
        ratio = (w / step.double()[:, None]).float().double().round().masked_fill(~some[:, None], 0.0)
        code = (ratio + zero[:, None]).clamp(0.0, 15.0)
        values[:, g0:g0 + group] = (code - zero[:, None]) * step.double()[:, None]
        scales.append(step.double())
        zeros.append(zero.long())
    return dict(scales=torch.stack(scales, 1), zeros=torch.stack(zeros, 1) if c["zeros"] else None, values=values)
