"""The operators of the two vocabulary-sized ends of a drafter, with their gradients.

`token_logprobs` and `embed_tokens` are binding.token_logprobs_raw and binding.embed_tokens_raw with
torch's autograd around them: where a gradient is wanted, the backward pass runs
binding.token_logprobs_backward and binding.embed_tokens_backward.  Nothing is computed here.

A step that is captured into a CUDA graph calls the forward and backward functions of the binding
directly: autograd nodes that were made outside a capture (a leaf's accumulation, say) would tie
their own stream into it, so a differentiable call during a capture is refused.
"""
import torch
from torch.autograd.function import once_differentiable

from . import binding


def _not_capturing():
    if torch.cuda.is_current_stream_capturing():
        raise binding.GlsError("a differentiable call can not be captured into a CUDA graph: capture the "
                               "forward and backward functions of the binding instead")


def _plain(g):
    return None if g is None else g.to(torch.float32).contiguous()


class _TokenLogprobs(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, tokens, top, kw):
        _not_capturing()
        dev, lead = logits.device, tuple(logits.shape[:3])
        tail = (0,) if tokens is None else tuple(tokens.shape[3:])
        f = dict(dtype=torch.float32, device=dev)
        out = dict(logprobs=torch.empty(lead + tail, **f), lse=torch.empty(lead, **f),
                   lse_tail=torch.empty(lead, **f))
        if kw["want_entropy"]:
            out["entropy"] = torch.empty(lead, **f)
        if top:
            out["top_ids"] = torch.empty(lead + (top,), dtype=torch.int32, device=dev)
            out["top_logprobs"] = torch.empty(lead + (top,), **f)
        binding.token_logprobs_raw(logits, tokens, top=top, out=out, **kw)
        ctx.kw = dict(inv_temp=kw["inv_temp"], inv_temp_per_draft=kw["inv_temp_per_draft"])
        ids = out.get("top_ids")
        ctx.save_for_backward(logits, tokens, out["lse"], out["lse_tail"], out.get("entropy"), ids)
        ctx.set_materialize_grads(False)
        if ids is not None:
            ctx.mark_non_differentiable(ids)
        return out["logprobs"], out["lse"], out.get("entropy"), ids, out.get("top_logprobs")

    @staticmethod
    @once_differentiable
    def backward(ctx, g_lp, g_lse, g_ent, _g_ids, g_top):
        _not_capturing()
        logits, tokens, lse, tail, ent, ids = ctx.saved_tensors
        grad = binding.token_logprobs_backward(
            logits, tokens, lse, entropy=ent, lse_tail=tail, top_ids=ids,
            grad_logprobs=_plain(g_lp) if tokens is not None else None, grad_lse=_plain(g_lse),
            grad_entropy=_plain(g_ent), grad_top_logprobs=_plain(g_top), **ctx.kw)
        return grad, None, None, None


def token_logprobs(logits, tokens, top=0, inv_temp=1.0, inv_temp_per_draft=None, want_entropy=True,
                   status=None, out=None):
    """Log probabilities of the tokens (int32 [B,K,J] or [B,K,J,G], -1: none) under the rows of logits
    [B,K,J,V], with the rows' log-sum-exp, entropy and `top` most likely tokens.

    Returns dict(logprobs, lse, entropy, top_ids, top_logprobs), the entropy only if wanted and the
    alternatives only for top > 0; see gls_token_logprobs in include/gls.h.  Differentiable in the
    logits (in reverse mode, once; not during a graph capture, and not into given outputs)."""
    if not (logits.requires_grad and torch.is_grad_enabled()):
        return binding.token_logprobs_raw(logits, tokens, top, inv_temp, inv_temp_per_draft, want_entropy, status, out)
    binding._no_tangent(logits)
    kw = dict(inv_temp=inv_temp, inv_temp_per_draft=inv_temp_per_draft, want_entropy=want_entropy,
              status=status)
    if out is not None:
        raise binding.GlsError("given outputs can not carry a gradient: call under torch.no_grad()")
    names = ("logprobs", "lse", "entropy", "top_ids", "top_logprobs")
    return {n: v for n, v in zip(names, _TokenLogprobs.apply(logits, tokens, binding._top(top), kw)) if v is not None}


class _EmbedTokens(torch.autograd.Function):
    @staticmethod
    def forward(ctx, table, tokens, scale, status):
        _not_capturing()
        ctx.save_for_backward(tokens)
        ctx.V, ctx.scale = table.shape[0], scale
        return binding.embed_tokens_raw(table, tokens, scale=scale, status=status)

    @staticmethod
    @once_differentiable
    def backward(ctx, g):
        _not_capturing()
        return binding.embed_tokens_backward(g, ctx.saved_tensors[0], ctx.V, scale=ctx.scale), None, None, None


def embed_tokens(table, tokens, scale=1.0, status=None, out=None):
    """scale * table[tokens]: table [V,D], int32 tokens of any shape -> [*tokens.shape, D]; a token
    below 0 gives zeros; see gls_embed_tokens in include/gls.h.  Differentiable in the table (in reverse
    mode, once; not during a graph capture, and not into a given output)."""
    if not (table.requires_grad and torch.is_grad_enabled()):
        return binding.embed_tokens_raw(table, tokens, scale, status, out)
    binding._no_tangent(table)
    if out is not None:
        raise binding.GlsError("a given output can not carry a gradient: call under torch.no_grad()")
    return _EmbedTokens.apply(table, tokens, float(scale), status)
