"""chgnet_embed_forward and chgnet_embed_backward against their definition in 64 bits (ops_reference.py): tables from one
row to many, tokens that are all one row, all different, outside the table; widths, types and strides; sizes around the
chunks, digits and passes of the ordering; streams and captured graphs."""
import pytest
import torch

import ops_reference as ref
from paper_2412_20796_amd import binding as bd
from paper_2412_20796_amd import ops

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def _tokens(n, vocab, first, how, seed=0):
    g = torch.Generator().manual_seed(17 * n + vocab + seed)
    if how == "one":
        t = torch.full((n,), vocab // 2)
    elif how == "two ends":
        t = torch.randint(0, 2, (n,), generator=g) * (vocab - 1)
    elif how == "in order":
        t = (torch.arange(n) * vocab) // max(n, 1)
    elif how == "none":
        t = torch.full((n,), -1 - first)
    elif how == "skewed":
        t = (torch.rand(n, generator=g, dtype=torch.float64) ** 6 * vocab).long().clamp_(max=vocab - 1)
    else:
        t = torch.randint(0, vocab, (n,), generator=g)
    t = t + first
    if how == "outside":
        far = torch.tensor([-1, first - 1, vocab + first, 2 ** 31 - 1, -2 ** 31])
        at = torch.rand(n, generator=g) < 0.3
        t = torch.where(at, far[torch.randint(0, 5, (n,), generator=g)], t)
    return t.to(torch.int32)


def _back(tok, dout, vocab, scale, first, **kw):
    return ops.embed_backward(tok.cuda(), dout.cuda(), vocab, scale=scale, first=first, **kw)


def _rand(n, d, dtype, seed=0):
    return torch.randn(n, d, generator=torch.Generator().manual_seed(n + d + seed)).to(dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,vocab,d", [(1, 1, 1), (1, 94, 64), (5, 94, 128), (8, 94, 64), (100, 7, 3), (257, 1000, 100),
                                       (1000, 94, 256), (33, 11, 333), (64, 5, 1024), (3, 2, 4097), (20000, 94, 64),
                                       (70001, 500, 12)])
def test_lookup(n, vocab, d, dtype):
    table = _rand(vocab, d, dtype)
    for how, first, scale in (("random", 0, 1.0), ("outside", 1, d ** 0.5), ("none", 0, 2.0)):
        tok = _tokens(n, vocab, first, how)
        got = ops.embed_forward(table.cuda(), tok.cuda(), scale=scale, first=first)
        assert torch.equal(got.cpu(), ref.embed(table, tok, scale, first)), how


def test_lookup_keeps_nan_and_infinity_in_their_rows():
    table = _rand(10, 64, torch.float32)
    table[3, 5], table[4, 6] = float("nan"), float("inf")
    tok = torch.tensor([3, 1, 4, -1, 3], dtype=torch.int32)
    got = ops.embed_forward(table.cuda(), tok.cuda(), scale=2.0).cpu()
    assert torch.equal(got.isnan(), ref.embed(table, tok, 2.0, 0).isnan()) and not bool(got[3].any())
    assert got[2, 6] == float("inf")


def test_lookup_strides():
    for dtype in TYPES:
        for d, pad, shift in ((64, 4, 0), (64, 1, 0), (30, 2, 1), (128, 0, 2)):
            big = _rand(50, d + pad, dtype)
            t = torch.empty(shift + 50 * (d + pad), dtype=dtype, device="cuda")[shift:].reshape(50, d + pad)
            t.copy_(big)
            out = torch.full((40, d + 3), 7.0, dtype=dtype, device="cuda")
            tok = _tokens(37, 50, 0, "outside")
            ops.embed_forward(t[:, :d], tok.cuda(), scale=0.5, out=out[:37, :d])
            assert torch.equal(out[:37, :d].cpu(), ref.embed(big[:, :d], tok, 0.5, 0))
            assert bool((out[37:] == 7).all()) and bool((out[:, d:] == 7).all())


# sizes below and above the switches to the ordering (16,384 tokens; 2^23 tokens looked at by row: 8,388 of 1,000 rows, and
# 2^22 by token: 2,023 of 3,000 rows; lanes: 12,288 of 128), around its stretches of 1,024 tokens a block, its chunks of 16 and more, digits of one to three passes, widths of one and several column blocks
@pytest.mark.parametrize("how", ["random", "one", "two ends", "in order", "outside", "none", "skewed"])
@pytest.mark.parametrize("n,vocab,d", [(1, 1, 1), (1, 94, 64), (63, 94, 64), (513, 94, 128), (1023, 3000, 20),
                                       (1024, 94, 128), (1025, 94, 128), (1040, 1, 64), (2047, 2, 64), (2048, 255, 130),
                                       (2049, 256, 65), (5844, 94, 128), (16384, 128, 64), (16384, 129, 64),
                                       (16385, 94, 64), (16383, 94, 130), (8388, 1000, 64), (8389, 1000, 64),
                                       (2023, 3000, 64), (2060, 3000, 64), (12288, 94, 128), (12289, 94, 128), (9999, 70000, 33), (16400, 300, 512),
                                       (40000, 1000, 9), (300007, 94, 64)])
def test_gradient(n, vocab, d, how):
    first = n % 2
    tok, dout = _tokens(n, vocab, first, how), _rand(n, d, torch.float32)
    r, b = ref.embed_grad(tok, dout, vocab, 0.75, first)
    ref.assert_within(_back(tok, dout, vocab, 0.75, first), r, b)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,vocab,d", [(700, 94, 64), (3000, 94, 128), (3000, 500, 256), (2000, 50, 77), (17000, 50, 77), (5000, 40, 1024),
                                       (17000, 40, 1024)])
def test_gradient_types(n, vocab, d, dtype):
    tok, dout = _tokens(n, vocab, 0, "skewed"), _rand(n, d, dtype)
    r, b = ref.embed_grad(tok, dout, vocab, d ** 0.5, 0)
    ref.assert_within(_back(tok, dout, vocab, d ** 0.5, 0), r, b)


def test_gradient_is_the_adjoint_of_the_lookup():
    """<lookup(W), y> = <W, gradient(y)>, and W's gradient by differences: the lookup is linear, so that a difference of
    any size is exact but for rounding."""
    n, vocab, d, scale = 2500, 94, 64, 1.5
    tok, W, y = _tokens(n, vocab, 1, "outside"), _rand(vocab, d, torch.float32), _rand(n, d, torch.float32, seed=1)
    g = _back(tok, y, vocab, scale, 1).cpu().double()
    out = lambda W: ops.embed_forward(W.cuda(), tok.cuda(), scale=scale, first=1).cpu().double()
    left, right = float((out(W) * y.double()).sum()), float((W.double() * g).sum())
    # one rounding of each product on the left, the gradient's bound on the right
    bound = float((scale * ref.U * W.abs().double()[ref.table_rows(tok, 1, vocab).clamp(max=vocab - 1)] * y.abs()).sum())
    bound += float((ref.embed_grad(tok, y, vocab, scale, 1)[1] * W.abs()).sum())
    assert abs(left - right) <= bound
    V = torch.zeros(vocab, d)
    V[7, 9] = 1.0
    assert abs(float((out(V) * y.double()).sum()) - float(g[7, 9])) <= float(
        ref.embed_grad(tok, y, vocab, scale, 1)[1][7, 9]) + scale * ref.U * float(y[:, 9].abs().sum())


@pytest.mark.parametrize("n", [0, 40, 1024, 1025, 6000, 20000])
def test_accumulate(n):
    vocab, d = 94, 64
    tok, dout = _tokens(n, vocab, 0, "skewed"), _rand(n, d, torch.float32)
    once = _back(tok, dout, vocab, 1.0, 0)
    base = torch.randn(vocab, d, device="cuda")
    got = _back(tok, dout, vocab, 1.0, 0, dtable=base.clone(), accumulate=True)
    # sum of the same two numbers, or product and sum in one rounding
    assert float((got.double() - (base.double() + once.double())).abs().max()) <= 2 * ref.U * float(
        (base.abs() + once.abs()).max())
    untouched = once.abs().sum(1) == 0
    assert torch.equal(got[untouched], base[untouched])
    if n == 0:
        assert not bool(once.any())


@pytest.mark.parametrize("n", [200, 3000, 17000])
def test_gradient_strides(n):
    vocab = 94
    for dtype in TYPES:
        for d, pad, shift in ((64, 4, 0), (64, 1, 0), (30, 2, 1), (128, 0, 2)):
            tok, dout = _tokens(n, vocab, 0, "random"), _rand(n, d, dtype)
            x = torch.empty(shift + n * (d + pad), dtype=dtype, device="cuda")[shift:].reshape(n, d + pad)
            x[:, :d].copy_(dout)
            out = torch.full((vocab + 2, d + pad + 3), 7.0, device="cuda")
            ops.embed_backward(tok.cuda(), x[:, :d], vocab, dtable=out[1:vocab + 1, :d])
            r, b = ref.embed_grad(tok, dout, vocab, 1.0, 0)
            ref.assert_within(out[1:vocab + 1, :d], r, b)
            assert bool((out[:, d:] == 7).all()) and bool((out[0] == 7).all()) and bool((out[vocab + 1] == 7).all())


@pytest.mark.parametrize("n", [500, 4000, 17000])
def test_gradient_of_values_that_are_not_finite(n):
    tok, dout = _tokens(n, 94, 0, "random"), _rand(n, 64, torch.float32)
    tok[n // 2] = 17
    clean = _back(tok, dout, 94, 1.0, 0).cpu()
    dout[n // 2, 11] = float("nan")
    got = _back(tok, dout, 94, 1.0, 0).cpu()
    assert bool(got[17, 11].isnan())
    got[17, 11] = clean[17, 11]
    assert torch.equal(got, clean)
    # a row outside the table does not matter, whatever it holds
    tok[n // 2] = -1
    assert bool(torch.isfinite(_back(tok, dout, 94, 1.0, 0)).all())


def test_large_table_and_offsets_past_32_bits():
    """Tokens of a table of 20,000,003 rows (four digits' passes), 2.56e9 values: rows past 2^31 values."""
    n, vocab, d = 5000, 20_000_003, 128
    tok = _tokens(n, vocab, 0, "random")
    tok[:3] = torch.tensor([vocab - 1, vocab - 1, 0], dtype=torch.int32)
    dout = _rand(n, d, torch.float32)
    dw = _back(tok, dout, vocab, 1.0, 0)
    got = ops.embed_forward(dw, tok.cuda())
    uniq, inv = torch.unique(tok.long(), return_inverse=True)
    want = torch.zeros(uniq.numel(), d, dtype=torch.float64).index_add_(0, inv, dout.double())
    ref.assert_within(got, want[inv], 2 * ref.U * 3 * dout.abs().double().max() * torch.ones(n, d))
    assert int((dw != 0).any(1).sum()) == uniq.numel()


@pytest.mark.parametrize("n", [900, 200003])
def test_bitwise_reproducible(n):
    tok, dout = _tokens(n, 94, 0, "skewed"), _rand(n, 128, torch.float32)
    assert torch.equal(_back(tok, dout, 94, 1.0, 0), _back(tok, dout, 94, 1.0, 0))


def test_captured_and_replayed():
    """Graphs of a few and of many tokens, replayed in turn with new tokens and eager calls between them."""
    s, made = torch.cuda.Stream(), []
    for n, vocab, d in ((300, 94, 64), (18000, 94, 128), (7000, 9000, 64)):
        x = dict(tok=_tokens(n, vocab, 0, "random").cuda(), dout=_rand(n, d, torch.float32).cuda(), ws=bd.Workspace(),
                 shape=(n, vocab, d), table=_rand(vocab, d, torch.float32).cuda())
        call = lambda x=x: (ops.embed_forward(x["table"], x["tok"], scale=3.0),
                            ops.embed_backward(x["tok"], x["dout"], x["shape"][1], scale=3.0, ws=x["ws"]))
        with torch.cuda.stream(s):
            call()
        torch.cuda.synchronize()
        x["graph"] = torch.cuda.CUDAGraph()
        with torch.cuda.graph(x["graph"], stream=s):
            x["out"], x["dw"] = call()
        made.append(x)
    for turn in range(3):
        for x in made:
            n, vocab, d = x["shape"]
            x["tok"].copy_(_tokens(n, vocab, 0, "outside", seed=turn))
            x["dout"].copy_(_rand(n, d, torch.float32, seed=turn))
            x["graph"].replay()
        torch.cuda.synchronize()
        for x in made:
            n, vocab, d = x["shape"]
            assert torch.equal(x["dw"], ops.embed_backward(x["tok"].clone(), x["dout"].clone(), vocab, scale=3.0))
            assert torch.equal(x["out"], ops.embed_forward(x["table"], x["tok"].clone(), scale=3.0))


@pytest.mark.parametrize("n", [500, 20000])
def test_two_streams_at_once(n):
    """Calls on two streams with workspaces of their own, and without any given, none waiting for the other."""
    vocab, d = 94, 128
    data = [(_tokens(n, vocab, 0, "skewed", seed=k).cuda(), _rand(n, d, torch.float32, seed=k).cuda()) for k in range(2)]
    want = [ops.embed_backward(t, x, vocab) for t, x in data]
    streams, ws = [torch.cuda.Stream() for _ in range(2)], [bd.Workspace(), None]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        for k, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[k].append(ops.embed_backward(*data[k], vocab, ws=ws[k]))
    torch.cuda.synchronize()
    for k in range(2):
        assert all(torch.equal(g, want[k]) for g in got[k])


def test_what_the_binding_refuses():
    table, tok, dout = torch.zeros(9, 8, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda"), torch.zeros(4, 8, device="cuda")
    for call in (lambda: ops.embed_forward(table, tok.long()), lambda: ops.embed_forward(table, tok.reshape(2, 2)),
                 lambda: ops.embed_forward(table.double(), tok), lambda: ops.embed_forward(table[0], tok),
                 lambda: ops.embed_forward(table, tok, first=-1), lambda: ops.embed_forward(table, tok, first=1 << 32),
                 lambda: ops.embed_forward(table, tok, out=torch.zeros(4, 7, device="cuda")),
                 lambda: ops.embed_forward(table, tok, out=torch.zeros(4, 8, device="cuda", dtype=torch.bfloat16)),
                 lambda: ops.embed_forward(table, tok.cpu()), lambda: ops.embed_forward(table.t(), tok),
                 lambda: ops.embed_forward(table[:0], tok), lambda: ops.embed_backward(tok, dout, 0),
                 lambda: ops.embed_backward(tok[:3], dout, 9), lambda: ops.embed_backward(tok, dout, 9, first=1 << 40),
                 lambda: ops.embed_backward(tok, dout[:1].expand(4, 8), 9),
                 lambda: ops.embed_backward(tok, dout, 9, accumulate=True),
                 lambda: ops.embed_backward(tok, dout, 9, dtable=torch.zeros(9, 8, device="cuda", dtype=torch.bfloat16)),
                 lambda: ops.embed_backward(tok, dout, 9, dtable=torch.zeros(8, 8, device="cuda")),
                 lambda: ops.embed_backward(torch.zeros(20000, dtype=torch.int32, device="cuda"),
                                            torch.zeros(20000, 8, device="cuda"), 9, ws=bd.Workspace("cpu"))):
        with pytest.raises(bd.ChgnetError) as e:
            call()
        assert e.value.code == bd.CHGNET_EINVAL


@pytest.mark.parametrize("n,vocab", [(300, 94), (300, 5000), (20000, 94), (20000, 70000)])
def test_rows_without_a_token_are_zero_at_any_scale(n, vocab):
    tok = _tokens(n, vocab, 0, "one").cuda()
    for scale in (-1.0, float("inf")):
        dw = ops.embed_backward(tok, torch.ones(n, 64, device="cuda"), vocab, scale=scale)
        assert bool((dw[vocab // 2] == scale * n).all())
        dw[vocab // 2] = 0
        assert torch.equal(dw.view(torch.int32), torch.zeros_like(dw).view(torch.int32))  # and no negative zeros
