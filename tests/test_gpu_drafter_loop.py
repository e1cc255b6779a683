"""The operators of a drafter's vocabulary ends run together, as pipeline.draft_position calls them: a 4-bit head and
embedding made from weights, logits, tokens, next inputs, position after position, then the verification."""
import numpy as np
import pytest
import torch

from paper_2506_05632_b200 import pipeline
from tests import vocab_ops_ref as ref

pytestmark = pytest.mark.gpu
B, K, L, V, D, SEED = 3, 4, 3, 5003, 96, 77


def _make(gls):
    g = torch.Generator(device="cuda").manual_seed(5)
    head = gls.quantize_table(0.2 * torch.randn((V, D), generator=g, device="cuda"), group=32)
    emb = gls.quantize_table(torch.randn((V, D), generator=g, device="cuda"), group=64, zeros=False, scale_dtype=torch.float32)
    mix = torch.randn((D, D), generator=g, device="cuda", dtype=torch.float32) / D ** 0.5
    first = torch.randn((B, 1, D), generator=g, device="cuda").expand(B, K, D).to(torch.bfloat16)
    return head, emb, mix.to(torch.bfloat16), first


def _body(x, mix):
    return torch.tanh(x @ mix) * 2.0


def _loop(buf, mix, first, **kw):
    x = first
    for j in range(L):
        u = kw.get("uniforms")
        x = pipeline.draft_position(_body(x, mix), j, buf, **dict(kw, **({} if u is None else dict(uniforms=u[j]))))
    return buf.draft_tokens


def test_drafts_by_the_races_and_their_verification(gls, oracle):
    head, emb, mix, first = _make(gls)
    buf = pipeline.DraftBuffers(B, K, L, head, emb)
    x = first
    for j in range(L):
        h = _body(x, mix)
        x = pipeline.draft_position(h, j, buf, inv_temp=1.25, seed=SEED)
        torch.cuda.synchronize()
        ref.check_logits(buf.logits.view(B * K, V), h.reshape(B * K, D), head)
        want = oracle.draft_sample(buf.logits.float().cpu().numpy(), seed=SEED, inv_temp=1.25, pos_base=j)
        assert np.array_equal(buf.tokens.cpu().numpy(), want["tokens"])
        assert torch.equal(buf.draft_tokens[:, :, j], buf.tokens[:, :, 0])
        assert torch.equal(x, ref.rows32(emb, 1.0, torch.bfloat16)[buf.tokens[:, :, 0].long()])
    target = (3.0 * torch.randn((B, K, L + 1, V), device="cuda")).to(torch.bfloat16)
    out = gls.target_sample_verify(target, buf.draft_tokens, seed=SEED, inv_temp=1.25)
    again = oracle.target_sample_verify(target.float().cpu().numpy(), buf.draft_tokens.cpu().numpy(), seed=SEED, inv_temp=1.25)
    assert np.array_equal(out["tokens"].cpu().numpy(), again["tokens"])
    assert int(buf.status) == 0


def test_independent_drafts(gls):
    head, emb, mix, first = _make(gls)
    buf = pipeline.DraftBuffers(B, K, L, head, emb, logits_dtype=torch.float32)
    u = torch.rand((L, B, K, 1), device="cuda")
    kw = dict(inv_temp=torch.tensor([1.0, 0.7, float("inf")], device="cuda"), top_k=50, top_p=0.9, min_p=0.01)
    x = first
    for j in range(L):
        x = pipeline.draft_position(_body(x, mix), j, buf, uniforms=u[j], **kw)
        tokens, lp = ref.sample(buf.logits, u[j], **kw)
        assert torch.equal(buf.tokens.cpu().long(), tokens)
        assert bool(((buf.scores.cpu().double() - lp).abs() <= ref.SLP + ref.U * lp.abs()).all())
    assert int(buf.status) == 0


@pytest.mark.parametrize("independent", [False, True])
def test_the_loop_as_a_graph(gls, independent):
    head, emb, mix, first = _make(gls)
    first = first.contiguous()
    kw = dict(uniforms=torch.rand((L, B, K, 1), device="cuda"), top_p=0.95) if independent else dict(seed=SEED)
    eager = pipeline.DraftBuffers(B, K, L, head, emb)
    buf = pipeline.DraftBuffers(B, K, L, head, emb)
    _loop(buf, mix, first, **kw)  # first use outside the capture
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _loop(buf, mix, first, **kw)
    for i in range(2):
        first.copy_(torch.randn((B, 1, D), device="cuda").expand(B, K, D))
        graph.replay()
        torch.cuda.synchronize()
        got = buf.draft_tokens.clone()
        assert torch.equal(got, _loop(eager, mix, first, **kw))


def test_two_graphs_and_an_eager_call_at_once(gls):
    """No workspace is shared: two captured loops and an eager one on streams of their own."""
    head, emb, mix, first = _make(gls)
    first = first.contiguous()
    bufs = [pipeline.DraftBuffers(B, K, L, head, emb) for _ in range(3)]
    u = torch.rand((L, B, K, 1), device="cuda")
    want = [_loop(b, mix, first, uniforms=u, top_k=k).clone() for b, k in zip(bufs, (5, 50, 500))]
    graphs = []
    for b, k in zip(bufs[:2], (5, 50)):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            _loop(b, mix, first, uniforms=u, top_k=k)
        graphs.append(graph)
    streams = [torch.cuda.Stream() for _ in range(3)]
    for b in bufs:
        b.draft_tokens.fill_(-9)
    torch.cuda.synchronize()
    for _ in range(5):
        for graph, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                graph.replay()
        with torch.cuda.stream(streams[2]):
            _loop(bufs[2], mix, first, uniforms=u, top_k=500)
    torch.cuda.synchronize()
    for b, w in zip(bufs, want):
        assert torch.equal(b.draft_tokens, w)


def test_a_plain_embedding_and_refusals(gls):
    head, _, mix, first = _make(gls)
    table = torch.randn((V, 40), device="cuda")
    buf = pipeline.DraftBuffers(B, K, 1, head, table, embed_scale=2.0)
    x = pipeline.draft_position(first, 0, buf, seed=SEED)
    assert torch.equal(x, 2.0 * table[buf.tokens[:, :, 0].long()])
    with pytest.raises(gls.GlsError):
        pipeline.draft_position(first, 1, buf)
    with pytest.raises(gls.GlsError):
        pipeline.draft_position(first, 0, buf, top_k=5)


def test_both_ways_of_a_call(gls, monkeypatch):
    """The compiled calls and the general way return the same, bit for bit, and refuse the same."""
    head, emb, mix, first = _make(gls)
    x = (2.0 * torch.randn((B, K, 1, V), device="cuda")).to(torch.bfloat16)
    u = torch.rand((B, K, 1), device="cuda")
    tok = torch.randint(-1, V, (4, 5), device="cuda", dtype=torch.int32)
    k = torch.randint(1, 90, (B, 1), device="cuda", dtype=torch.int32)

    def run():
        a = gls.sample_tokens(x, u, top_k=k, top_p=0.9, inv_temp=1.5)
        return [a["tokens"], a["logprobs"], gls.sample_tokens(x, u, want_logprobs=False)["tokens"],
                gls.head_logits(first, head), gls.head_logits(first, head, dtype=torch.float32),
                gls.embed_tokens_int4(emb, tok, scale=0.5), gls.embed_tokens_int4(emb, tok, dtype=torch.float32)]

    def refused():
        n = 0
        for call in (lambda: gls.sample_tokens(x, u, top_p=-1.0), lambda: gls.sample_tokens(x, u[:1]),
                     lambda: gls.head_logits(first[..., :5], head), lambda: gls.embed_tokens_int4(emb, tok.long()),
                     lambda: gls.embed_tokens_int4(emb._replace(dim=95), tok, scale=float("inf"))):
            with pytest.raises(gls.GlsError):
                call()
            n += 1
        return n

    one, r1 = run(), refused()
    monkeypatch.setattr(gls.binding, "_calls", gls.binding._GeneralWay())
    two, r2 = run(), refused()
    assert r1 == r2 and all(a.dtype is b.dtype and torch.equal(a, b) for a, b in zip(one, two))
