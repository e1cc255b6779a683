"""4-bit tables: made from weights (codes, scales and zeros equal to the definition's), read by token (equal) and
multiplied with hidden states (within the tolerance derived in vocab_ops_ref.py)."""
import pytest
import torch

from tests import vocab_ops_ref as ref

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _weights(V, D, dtype, seed):
    return (0.05 * torch.randn((V, D), generator=_gen(seed), device="cuda")).to(dtype)


def _table(gls, V, D, group, zeros, scale_dtype, seed):
    """A table as another program may have written it: any codes, zeros whose high bits are set, rows further apart."""
    g = _gen(seed)
    G, pitch = -(-D // group), -(-D // 32) * 16
    codes = torch.randint(0, 256, (V, pitch + 16), generator=g, device="cuda", dtype=torch.uint8)[:, :pitch]
    scales = ((torch.rand((V, G + 3), generator=g, device="cuda") - 0.3) * 0.1).to(scale_dtype)[:, :G]
    z = torch.randint(0, 256, (V, G), generator=g, device="cuda", dtype=torch.uint8) if zeros else None
    return gls.Int4Table(codes, scales, z, D, group)


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("dtype,scale_dtype", [(F32, F32), (F32, BF16), (BF16, BF16), (BF16, F32)])
def test_quantize(gls, group, zeros, dtype, scale_dtype):
    for V, D in ((1, 1), (3, 31), (17, 64), (5, 129), (40, 1000), (9, 4099), (300, 256)):
        w = _weights(V, D, dtype, V * D)
        t = gls.quantize_table(w, group=group, zeros=zeros, scale_dtype=scale_dtype)
        q, s, z = ref.quantize(w, group, zeros, scale_dtype)
        codes, tz = ref.unpack(t)
        assert torch.equal(t.scales.double(), s), (V, D)
        assert torch.equal(tz, z) and torch.equal(codes, q), (V, D)
        if D % 2:
            assert bool((t.codes[:, D // 2] >> 4 == 0).all())


def test_quantize_ties_and_extremes(gls):
    w = torch.zeros((9, 64), device="cuda")
    w[0, :32] = torch.arange(32, device="cuda") * 0.5 - 4.0    # quotients on half steps
    w[1, :] = 7.0
    w[2, :] = -7.0
    w[3, 3] = float("inf")
    w[4, 40] = float("nan")
    w[5, 5] = torch.finfo(F32).max
    w[6, :4] = torch.tensor([1e-42, -1e-42, 3e-41, 1e-45], device="cuda")
    w[7, 7] = -torch.finfo(F32).max
    w[7, 8] = torch.finfo(F32).max
    w[8, ::2] = 1e-30
    for zeros in (False, True):
        for sd in (F32, BF16):
            t = gls.quantize_table(w, group=32, zeros=zeros, scale_dtype=sd)
            q, s, z = ref.quantize(w, 32, zeros, sd)
            codes, tz = ref.unpack(t)
            assert torch.equal(t.scales.double().nan_to_num(-1.0), s.nan_to_num(-1.0)), (zeros, sd)
            assert torch.equal(codes, q) and torch.equal(tz, z), (zeros, sd)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_quantize_strides(gls, dtype):
    store = _weights(33, 517, dtype, 3)
    for w in (store[:, 1:401], store[::2, 3:100], store[:, 8:408]):
        t = gls.quantize_table(w, group=64)
        q, s, z = ref.quantize(w, 64, True, BF16)
        codes, tz = ref.unpack(t)
        assert torch.equal(codes, q) and torch.equal(tz, z) and torch.equal(t.scales.double(), s)


def test_quantize_into_given_tensors(gls):
    w = _weights(20, 100, BF16, 4)
    codes = torch.full((20, 96), 0xAB, dtype=torch.uint8, device="cuda")
    scales = torch.full((20, 7), 5.0, device="cuda")
    zeros = torch.full((20, 5), 77, dtype=torch.uint8, device="cuda")
    t = gls.quantize_table(w, out=gls.Int4Table(codes[:, 16:80], scales[:, :4], zeros[:, :4], 100, 32))
    q, s, z = ref.quantize(w, 32, True, F32)
    c, tz = ref.unpack(t)
    assert torch.equal(c, q) and torch.equal(tz, z) and torch.equal(t.scales.double(), s)
    assert bool((codes[:, :16] == 0xAB).all()) and bool((codes[:, 16 + 50:] == 0xAB).all())
    assert bool((scales[:, 4:] == 5.0).all()) and bool((zeros[:, 4:] == 77).all())


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_embed(gls, group, dtype):
    for V, D, zeros, sd in ((50, 1, True, BF16), (7, 77, False, F32), (300, 128, True, F32), (64, 1000, False, BF16), (11, 4100, True, BF16)):
        t = _table(gls, V, D, group, zeros, sd, V + D)
        tok = torch.randint(-1, V, (3, 41), generator=_gen(D), device="cuda", dtype=torch.int32)
        for scale in (1.0, 0.37):
            got = gls.embed_tokens_int4(t, tok, scale=scale, dtype=dtype)
            want = ref.rows32(t, scale, dtype)[tok.clamp(min=0).long()] * (tok >= 0)[..., None]
            assert got.shape == (3, 41, D) and torch.equal(got, want.to(dtype)), (V, D, scale)


def test_embed_tokens_outside_the_table_and_given_output(gls):
    t = _table(gls, 10, 70, 32, True, F32, 1)
    tok = torch.tensor([3, 10, -1, 1 << 30, -(1 << 31), 9], dtype=torch.int32, device="cuda")
    store = torch.full((6, 75), 9.0, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    gls.embed_tokens_int4(t, tok, out=store[:, 2:72], status=status)
    rows = ref.rows32(t, 1.0, F32)
    assert torch.equal(store[0, 2:72], rows[3]) and torch.equal(store[5, 2:72], rows[9])
    assert bool((store[1:5, 2:72] == 0).all()) and bool((store[:, :2] == 9).all()) and bool((store[:, 72:] == 9).all())
    assert int(status) == gls.DEV_BAD_TOKEN
    assert gls.embed_tokens_int4(t, tok[:0]).shape == (0, 70)


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("xt", [F32, BF16])
def test_head(gls, group, xt):
    i = 0
    for V, D in ((1, 1), (15, 33), (16, 128), (100, 500), (333, 1024), (1000, 2056), (257, 8192), (4099, 320)):
        for N in (1, 2, 5, 8, 9, 17, 64):
            i += 1
            t = _table(gls, V, D, group, i % 2 == 0, [F32, BF16][i % 3 == 0], i)
            x = torch.randn((N, D), generator=_gen(i), device="cuda").to(xt)
            got = gls.head_logits(x, t, dtype=[F32, BF16][i % 5 == 0])
            ref.check_logits(got, x, t, "%d x %d, N %d" % (V, D, N))


@pytest.mark.parametrize("xt", [F32, BF16])
def test_head_of_the_widest_rows(gls, xt):
    t = _table(gls, 50, 32768, 64, True, BF16, 2)
    x = torch.randn((3, 32768), generator=_gen(2), device="cuda").to(xt)
    ref.check_logits(gls.head_logits(x, t, dtype=F32), x, t)


@pytest.mark.parametrize("xt", [F32, BF16])
def test_head_of_many_hidden_states(gls, xt):
    for V, D, N, group in ((300, 130, 65, 128), (257, 1000, 130, 64), (5000, 96, 200, 32), (128, 8192, 24, 32), (1, 5, 9, 128),
                           (40000, 160, 40, 64), (130, 128, 64, 128)):
        for zeros in (False, True):
            t = _table(gls, V, D, group, zeros, [F32, BF16][N % 2], V + N)
            x = torch.randn((N, D), generator=_gen(N), device="cuda").to(xt)
            room = torch.full((N, V + 5), 3.0, device="cuda")
            gls.head_logits(x, t, out=room[:, 2:V + 2])
            ref.check_logits(room[:, 2:V + 2], x, t, str((V, D, N, group, zeros)))
            assert bool((room[:, :2] == 3).all()) and bool((room[:, V + 2:] == 3).all())


def test_head_workspace(gls):
    """A given workspace is used whatever it holds; one that is too small is refused; hidden states that lie anywhere."""
    t = _table(gls, 700, 333, 32, True, BF16, 21)
    store = torch.randn((20, 400), generator=_gen(21), device="cuda").to(BF16)
    n = gls.head_logits_workspace_bytes(20, 333, BF16)
    ws = torch.full((n + 64,), 0xFF, dtype=torch.uint8, device="cuda")
    for off in (0, 1, 7):
        x = store[:, off:off + 333]
        ref.check_logits(gls.head_logits(x, t, workspace=ws), x, t)
    with pytest.raises(gls.GlsError):
        gls.head_logits(x, t, workspace=ws[:n - 16])


def test_head_of_large_vocabularies(gls):
    for V, D, N, group in ((50257, 1000, 3, 32), (128256, 256, 8, 128), (32000, 1024, 1, 64), (20000, 2048, 33, 128)):
        t = _table(gls, V, D, group, True, BF16, V)
        x = torch.randn((N, D), generator=_gen(V), device="cuda").to(BF16)
        ref.check_logits(gls.head_logits(x, t, dtype=F32), x, t, str((V, D, N)))


def test_head_hidden_states_of_all_magnitudes(gls):
    t = _table(gls, 64, 256, 128, True, F32, 8)
    x = torch.randn((4, 256), generator=_gen(8), device="cuda")
    x[0] *= 1e30
    x[1] *= 1e-30
    x[2] = 0.0
    x[3, ::2] *= 2.0 ** 20
    ref.check_logits(gls.head_logits(x, t), x, t)
    y = x.clone()
    y[0, 5] = float("nan")
    y[2, 7] = float("inf")
    got = gls.head_logits(y, t)
    assert bool(torch.isnan(got[0]).all())
    w = ref.rows64(t)[:, 7]
    assert torch.equal(got[2], (w * float("inf")).float().nan_to_num(nan=float("nan"), posinf=float("inf"), neginf=float("-inf"))) or \
        torch.equal(torch.isnan(got[2]), w == 0)
    ref.check_logits(got[[1, 3]], x[[1, 3]], t)  # other rows do not feel it


def test_head_shapes_strides_and_given_output(gls):
    t = _table(gls, 200, 96, 32, False, BF16, 9)
    store = torch.randn((2, 3, 200), generator=_gen(9), device="cuda").to(BF16)
    x = store[..., 5:101]
    got = gls.head_logits(x, t)
    assert got.shape == (2, 3, 200) and got.dtype is BF16
    ref.check_logits(got, x, t)
    ref.check_logits(gls.head_logits(x.transpose(0, 1), t, dtype=F32), x.transpose(0, 1), t)
    one = store[0, 0, :96]
    ref.check_logits(gls.head_logits(one, t), one, t)
    wide = store[:1, :1, :96].expand(2, 3, 96)
    ref.check_logits(gls.head_logits(wide, t), wide, t)
    room = torch.full((6, 211), 3.0, device="cuda")
    out = room[:, 4:204].view(2, 3, 200)
    assert gls.head_logits(x, t, out=out) is out
    ref.check_logits(out, x, t)
    assert bool((room[:, :4] == 3).all()) and bool((room[:, 204:] == 3).all())
    assert gls.head_logits(x[:0], t).shape == (0, 3, 200)


def test_equal_calls_return_equal_bits_on_any_stream_and_in_graphs(gls):
    t = _table(gls, 3000, 1024, 128, True, BF16, 10)
    x = torch.randn((8, 1024), generator=_gen(10), device="cuda").to(BF16)
    want = gls.head_logits(x, t, dtype=F32)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = gls.head_logits(x, t, dtype=F32)
    side.synchronize()
    assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = gls.head_logits(x, t, dtype=F32)
    x.copy_(torch.randn((8, 1024), generator=_gen(11), device="cuda"))
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(held, gls.head_logits(x, t, dtype=F32))


def test_refusals(gls):
    t = _table(gls, 64, 100, 32, True, BF16, 12)
    x = torch.randn((2, 100), device="cuda").to(BF16)
    tok = torch.zeros(3, dtype=torch.int32, device="cuda")
    E = gls.GlsError
    for bad in (x[:, :99], x.cpu(), x.half(), x.clone().requires_grad_()):
        with pytest.raises(E):
            gls.head_logits(bad, t)
    for bad in (t._replace(codes=t.codes[:, :48]), t._replace(codes=t.codes.int()), t._replace(scales=t.scales[:, :3]),
                t._replace(scales=t.scales.half()), t._replace(zeros=t.zeros[:, :1]), t._replace(zeros=t.zeros.int()),
                t._replace(group=16), t._replace(group=0), t._replace(zeros=t.zeros.cpu()), t._replace(codes=t.codes.cpu())):
        with pytest.raises(E):
            gls.head_logits(x, bad)
        with pytest.raises(E):
            gls.embed_tokens_int4(bad, tok)
    with pytest.raises(E):
        gls.head_logits(x, t, dtype=torch.float16)
    with pytest.raises(E):
        gls.head_logits(x, t, out=torch.empty((2, 63), device="cuda"))
    shared = torch.zeros((64, 160), dtype=torch.uint8, device="cuda")
    inside = gls.Int4Table(shared[:, :64], t.scales, t.zeros, 100, 32)
    with pytest.raises(E):
        gls.head_logits(x, inside, out=shared.view(-1)[:2 * 64 * 2].view(BF16).view(2, 64))
    with pytest.raises(E):
        gls.embed_tokens_int4(t, tok.long())
    with pytest.raises(E):
        gls.embed_tokens_int4(t, tok, scale=float("nan"))
    with pytest.raises(E):
        gls.embed_tokens_int4(t, tok, dtype=torch.float16)
    w = torch.randn((64, 100), device="cuda")
    for kw in (dict(group=48), dict(scale_dtype=torch.float16), dict(out=t._replace(dim=96))):
        with pytest.raises(E):
            gls.quantize_table(w, **kw)
    for bad in (w.half(), w.T, w[0], w.cpu(), w.clone().requires_grad_()):
        with pytest.raises(E):
            gls.quantize_table(bad)


def test_quantize_quotients_of_all_sizes(gls):
    """Quotients next to half way between two codes, for steps of every mantissa: equal to those of a division."""
    g = _gen(77)
    step = (1.0 + torch.rand((4000, 1), generator=g, device="cuda")) * 2.0 ** torch.randint(-60, 60, (4000, 1), generator=g, device="cuda").float()
    k = torch.randint(-7, 7, (4000, 64), generator=g, device="cuda") + 0.5
    w = k * step * (1.0 + torch.randint(-3, 4, (4000, 64), generator=g, device="cuda") * 2.0 ** -23)
    w[:, 0] = 7.0 * step[:, 0]
    for zeros in (False, True):
        for x in (w, w.to(BF16)):
            for sd in (F32, BF16):
                t = gls.quantize_table(x, group=64, zeros=zeros, scale_dtype=sd)
                q, s, z = ref.quantize(x, 64, zeros, sd)
                codes, tz = ref.unpack(t)
                assert torch.equal(t.scales.double(), s) and torch.equal(tz, z) and torch.equal(codes, q), (zeros, x.dtype, sd)
