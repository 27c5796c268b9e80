"""chgnet_dropout against its definition, bit for bit: types, widths and rows around the generator's groups, strides, rates,
seeds and numbers of 64 bits, values that are not finite, streams and replayed graphs."""
import pytest
import torch

import block_reference as ref
from paper_2412_20796_amd import binding as bd
from paper_2412_20796_amd import ops

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def _x(rows, d, dtype, seed=0):
    g = torch.Generator().manual_seed(rows + 31 * d + seed)
    return torch.randn(rows, d, generator=g).to(dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,d", [(1, 1), (3, 7), (5, 8), (2, 9), (64, 64), (37, 100), (257, 333), (1, 5000), (3000, 16),
                                    (1200, 1001), (20000, 72)])
def test_sizes(rows, d, dtype):
    x = _x(rows, d, dtype)
    assert torch.equal(ops.dropout(x.cuda(), 0.3, 99, 5).cpu(), ref.dropout(x, 0.3, 99, 5))


@pytest.mark.parametrize("p", [0.0, 2.0 ** -17, 2.0 ** -16, 0.1, 0.5, 0.999, 1.0 - 2.0 ** -17, 1.0])
def test_rates(p):
    x = _x(300, 96, torch.float32)
    out = ops.dropout(x.cuda(), p, 1, 2).cpu()
    assert torch.equal(out, ref.dropout(x, p, 1, 2))
    if p == 0.0:
        assert torch.equal(out, x)
    if p == 1.0:
        assert not out.any()


@pytest.mark.parametrize("seed,call,step", [(0, 0, None), (2 ** 64 - 1, 2 ** 64 - 1, None), (1 << 40, 1 << 35, 3),
                                            (5, 2 ** 64 - 2, 7), (5, 10, -3)])
def test_seeds_and_numbers(seed, call, step):
    x = _x(33, 40, torch.float32)
    s = None if step is None else torch.tensor([step], device="cuda")
    want = ref.dropout(x, 0.5, seed, call + (step or 0))
    assert torch.equal(ops.dropout(x.cuda(), 0.5, seed, call, s).cpu(), want)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d,pad,shift", [(64, 8, 0), (64, 3, 0), (64, 8, 1), (50, 14, 0), (13, 0, 5)])
def test_strides_and_what_lies_between(d, pad, shift, dtype):
    rows = 41
    x = _x(rows, d, dtype)
    make = lambda: torch.full((shift + rows * (d + pad) + 9,), 7.0, dtype=dtype, device="cuda")
    view = lambda b: b[shift:shift + rows * (d + pad)].reshape(rows, d + pad)[:, :d]
    bx, bo = make(), make()
    view(bx).copy_(x)
    ops.dropout(view(bx), 0.4, 3, 4, out=view(bo))
    assert torch.equal(view(bo).cpu(), ref.dropout(x, 0.4, 3, 4))
    view(bo).fill_(7.0)
    assert bool((bo == 7).all())


def test_dropped_values_that_are_not_finite_are_zero():
    m, _ = ref.kept(50, 64, 0.5, 1, 1)
    x = torch.where(m, torch.ones(()), torch.tensor(float("nan")))
    x[~m & (torch.arange(64) % 2 == 0)] = float("inf")
    out = ops.dropout(x.cuda(), 0.5, 1, 1).cpu()
    assert torch.equal(out, ref.dropout(x, 0.5, 1, 1)) and bool(torch.isfinite(out).all())


def test_the_same_call_is_the_gradient():
    x, up = _x(70, 90, torch.float32), _x(70, 90, torch.float32, 1)
    a, b = (ops.dropout(t.cuda(), 0.2, 8, 9).cpu() for t in (x, up))
    assert torch.equal(a != 0, (b != 0) | (up == 0) & (a != 0))
    # linear in x: differences are exact products with the factor
    m, f = ref.kept(70, 90, 0.2, 8, 9)
    assert torch.equal(b, torch.where(m, up * torch.tensor(f, dtype=torch.float32), torch.zeros(())))


def test_empty():
    assert ops.dropout(torch.empty(0, 64, device="cuda"), 0.5, 1).shape == (0, 64)


def test_another_stream_and_two_at_once():
    x = _x(5000, 256, torch.bfloat16).cuda()
    want = [ref.dropout(x.cpu(), 0.1, s, 0) for s in (1, 2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in want]
    outs = []
    for k, s in enumerate(streams):
        with torch.cuda.stream(s):
            outs.append(ops.dropout(x, 0.1, k + 1))
    torch.cuda.synchronize()
    assert all(torch.equal(a.cpu(), b) for a, b in zip(outs, want))


def test_a_replayed_graph_draws_anew():
    x = _x(130, 200, torch.float32)
    xc, step = x.cuda(), torch.zeros(1, dtype=torch.int64, device="cuda")
    ops.dropout(xc, 0.5, 6, 100, step)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = ops.dropout(xc, 0.5, 6, 100, step)
        step.add_(1)
    for k in range(4):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out.cpu(), ref.dropout(x, 0.5, 6, 100 + k)), k
        assert float(x.sum()) == float(xc.cpu().sum())


def test_sizes_past_32_bits():
    rows, d = 70000, 32776
    x = torch.ones(rows, d, dtype=torch.bfloat16, device="cuda")
    out = ops.dropout(x, 0.5, 7, 1)
    for r in (0, 40000, 65535, rows - 1):
        n = ref.kept(1, d, 0.5, 7, 1)[0] if r == 0 else None
        got = out[r].cpu()
        if n is not None:
            assert torch.equal(got != 0, n[0])
        g = ref.philox(range((d + 7) // 8), [r] * ((d + 7) // 8), [1] * ((d + 7) // 8), [0] * ((d + 7) // 8), 7, 0)
        low, high = [(w.astype('int64') & 0xFFFF) >= 32768 for w in g], [(w.astype('int64') >> 16) >= 32768 for w in g]
        want = torch.tensor([v for k in range(len(low[0])) for i in range(4) for v in (low[i][k], high[i][k])])[:d]
        assert torch.equal(got != 0, want), r


def test_refusals():
    x = torch.zeros(4, 8, device="cuda")
    for call in (lambda: ops.dropout(x, 1.5, 0), lambda: ops.dropout(x, float("nan"), 0), lambda: ops.dropout(x, 0.1, -1),
                 lambda: ops.dropout(x, 0.1, 1 << 64), lambda: ops.dropout(x, 0.1, 0, -1), lambda: ops.dropout(x.T[:3], 0.1, 0),
                 lambda: ops.dropout(x, 0.1, 0, 0, torch.zeros(1, device="cuda")), lambda: ops.dropout(x[0], 0.1, 0),
                 lambda: ops.dropout(x, 0.1, 0, out=torch.zeros(4, 9, device="cuda"))):
        with pytest.raises(bd.ChgnetError) as e:
            call()
        assert e.value.code == bd.CHGNET_EINVAL
