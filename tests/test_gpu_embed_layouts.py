"""Layouts of the embedding kernels that only alignment, width or size select: rows with a stride of their own in vector
loads, four values a lane of 16-bit rows, the widest one-launch form, rows read past the caches, tables wider than one turn
of the join; each against the definition in 64 bits (ops_reference.py)."""
import pytest
import torch

import ops_reference as ref
from paper_2412_20796_amd import ops

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def _tokens(n, vocab, skew, seed=0):
    """skew: nine tenths on one row."""
    g = torch.Generator().manual_seed(3 * n + vocab + seed)
    t = torch.randint(-1, vocab + 1, (n,), generator=g)
    if skew:
        t = torch.where(torch.rand(n, generator=g) < 0.9, torch.full_like(t, vocab // 3), t)
    return t.to(torch.int32)


def _rand(n, d, dtype, seed=0):
    return torch.randn(n, d, generator=torch.Generator().manual_seed(n + d + seed)).to(dtype)


def _sums(tok, dout, vocab, scale):
    """The sums in 64 bits and a bound of fp32's roundings, from the longest chain of additions that a sum of m rows goes
    through. One launch: m / 16 rows in one of at least 16 groups of lanes, then the groups (64 at most). Ordered: 256 rows of
    a chunk at most, the chunks of a block (32), the blocks' partial rows, of 128 positions at least, by one group of lanes at
    least, then the groups (32). Never more than m. And the product with the scale, and a sum with what was there."""
    r = ref.table_rows(tok, 0, vocab)
    x = dout.double()
    s = torch.zeros(vocab + 1, x.shape[1], dtype=torch.float64).index_add_(0, r, x)[:vocab]
    a = torch.zeros(vocab + 1, x.shape[1], dtype=torch.float64).index_add_(0, r, x.abs())[:vocab]
    m = torch.bincount(r, minlength=vocab + 1)[:vocab, None].double()
    chain = torch.minimum(m, torch.maximum(m / 16 + 65, 256 + 32 + m / 128 + 2 + 32))
    return scale * s, 1.01 * abs(scale) * a * ref.U * (chain + 2)


def _aligned(rows, cols, ld, dtype, fill=7.0):
    """(buffer, view) of rows x cols values with a row stride of ld, its first value on a 16-byte boundary."""
    buf = torch.full((rows + 2, ld), fill, dtype=dtype, device="cuda")
    assert buf.data_ptr() % 16 == 0 and ld * buf.element_size() % 8 == 0
    return buf, buf[:rows, :cols]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d,pad", [(64, 8), (64, 4), (128, 8), (256, 12), (512, 8), (100, 4), (68, 8), (260, 4)])
def test_lookup_strides_of_vector_loads(d, pad, dtype):
    table, tok = _rand(50, d, dtype), _tokens(37, 50, False)
    _, tv = _aligned(50, d, d + pad, dtype)
    tv.copy_(table)
    for out_pad in (0, pad, pad + 4):
        buf, out = _aligned(37, d, d + out_pad, dtype)
        ops.embed_forward(tv, tok.cuda(), scale=0.5, out=out)
        assert torch.equal(out.cpu(), ref.embed(table, tok, 0.5, 0))
        assert bool((buf[37:] == 7).all()) and bool((buf[:, d:] == 7).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d,pad", [(64, 8), (64, 4), (128, 8), (256, 12), (512, 8), (100, 4), (68, 8), (260, 4)])
@pytest.mark.parametrize("n", [200, 3000, 17000])
def test_gradient_strides_of_vector_loads(n, d, pad, dtype):
    """One launch by row and by token (94 and 400 rows), and the ordering; overwritten and added to."""
    dout = _rand(n, d, dtype)
    _, x = _aligned(n, d, d + pad, dtype)
    x.copy_(dout)
    for vocab in (94, 400):
        tok = _tokens(n, vocab, False)
        r, b = _sums(tok, dout, vocab, 0.75)
        for add in (False, True):
            buf, dw = _aligned(vocab, d, d + pad, torch.float32)
            ops.embed_backward(tok.cuda(), x, vocab, scale=0.75, dtable=dw, accumulate=add)
            base = 7.0 if add else 0.0
            ref.assert_within(dw, r + base, b + 2 * ref.U * (base + r.abs()), what="vocab %d add %d" % (vocab, add))
            assert bool((buf[vocab:] == 7).all()) and bool((buf[:, d:] == 7).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("skew", [False, True])
@pytest.mark.parametrize("n,vocab,d", [(1000, 94, 512),             # one launch, 64 lanes of 16 bytes
                                       (3071, 94, 512), (6144, 94, 260),  # about as many tokens as that takes, 384 rows a group
                                       (1000, 94, 68), (20000, 94, 68), (1000, 94, 100), (20000, 94, 100),
                                       (1000, 94, 260), (20000, 94, 260), (2000, 9000, 68),
                                       (1000, 94, 2052), (300, 20, 4097), (3, 2, 65536), (40, 50, 65533)])
def test_gradient_layouts(n, vocab, d, skew, dtype):
    tok, dout = _tokens(n, vocab, skew), _rand(n, d, dtype)
    r, b = _sums(tok, dout, vocab, 1.5)
    ref.assert_within(ops.embed_backward(tok.cuda(), dout.cuda(), vocab, scale=1.5), r, b)


@pytest.mark.parametrize("n,vocab,d,dtype", [(20000, 30, 2052, torch.float32), (20000, 30, 2052, torch.bfloat16),
                                             (17000, 30, 4097, torch.bfloat16), (17000, 30, 4100, torch.float16)])
def test_join_takes_wide_rows_in_turns(n, vocab, d, dtype):
    """Runs over many blocks, of rows wider than the 2,048 (without vector loads 512) columns that the join takes at once."""
    tok, dout = _tokens(n, vocab, True), _rand(n, d, dtype)
    r, b = _sums(tok, dout, vocab, 1.0)
    ref.assert_within(ops.embed_backward(tok.cuda(), dout.cuda(), vocab), r, b)


@pytest.mark.parametrize("skew", [False, True])
@pytest.mark.parametrize("n,vocab,d,dtype", [(270001, 94, 128, torch.float32), (270001, 94, 256, torch.bfloat16),
                                             (530003, 20, 132, torch.float16), (140001, 3000, 256, torch.float32)])
def test_rows_read_past_the_caches(n, vocab, d, dtype, skew):
    """Rows of 128 MB and more."""
    assert n * d * dout_bytes(dtype) >= 128 << 20
    tok, dout = _tokens(n, vocab, skew), _rand(n, d, dtype)
    r, b = _sums(tok, dout, vocab, 0.5)
    dc = dout.cuda()
    got = ops.embed_backward(tok.cuda(), dc, vocab, scale=0.5)
    ref.assert_within(got, r, b)
    base = torch.randn(vocab, d)
    ref.assert_within(ops.embed_backward(tok.cuda(), dc, vocab, scale=0.5, dtable=base.cuda(), accumulate=True), base.double() + r,
                      b + 2 * ref.U * (base.double().abs() + r.abs()))
    assert torch.equal(got, ops.embed_backward(tok.cuda(), dc, vocab, scale=0.5))


def dout_bytes(dtype):
    return torch.empty(0, dtype=dtype).element_size()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,vocab,d", [(5, 3, 65536), (5, 3, 65535), (70, 9, 2052), (33, 7, 68), (70, 9, 260)])
def test_lookup_of_wide_and_unusual_rows(n, vocab, d, dtype):
    table, tok = _rand(vocab, d, dtype), _tokens(n, vocab, False)
    assert torch.equal(ops.embed_forward(table.cuda(), tok.cuda(), scale=3.0).cpu(), ref.embed(table, tok, 3.0, 0))
