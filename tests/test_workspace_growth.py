"""A workspace that grows after a captured call was given its buffer."""
import gc
import weakref

import pytest
import torch

from paper_2412_20796_amd import binding as bd
from paper_2412_20796_amd import ops

gpu = pytest.mark.gpu


def test_a_captured_workspace_outlives_its_growth(monkeypatch):
    """A buffer that a captured call was given stays allocated when the workspace grows: the graph writes to it at each
    replay. One that only eager calls had is given back."""
    capturing = [False]
    monkeypatch.setattr(bd, "_capturing", lambda buf: capturing[0], raising=False)
    ws = bd.Workspace("cpu")
    eager = weakref.ref(ws.ensure(100))
    ws.ensure(200)
    gc.collect()
    assert eager() is None
    capturing[0] = True
    captured = weakref.ref(ws.ensure(150))
    capturing[0] = False
    assert ws.ensure(180) is captured()
    ws.ensure(300)
    gc.collect()
    assert captured() is not None and captured().numel() == 200
    # also where the call takes the buffer as it is, as a backward pass does
    capturing[0], given = True, weakref.ref(ws.buf)
    ws.ptr
    capturing[0] = False
    ws.ensure(350)
    gc.collect()
    assert given() is not None
    later = weakref.ref(ws.ensure(350))
    ws.ensure(400)
    gc.collect()
    assert later() is None and captured() is not None
    del ws
    gc.collect()
    assert captured() is None


@gpu
def test_replay_after_the_workspace_has_grown():
    """The replayed graph does not write into tensors made after the growth."""
    vocab, d = 94, 64
    g = torch.Generator().manual_seed(4)
    tok = [torch.randint(0, vocab, (n,), generator=g, dtype=torch.int32).cuda() for n in (20000, 300000)]
    x = [torch.randn(t.numel(), d, generator=g).cuda() for t in tok]
    want = ops.embed_backward(tok[0], x[0], vocab)
    s, ws = torch.cuda.Stream(), bd.Workspace()
    with torch.cuda.stream(s):
        ops.embed_backward(tok[0], x[0], vocab, ws=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        out = ops.embed_backward(tok[0], x[0], vocab, ws=ws)
    small = ws.nbytes
    ops.embed_backward(tok[1], x[1], vocab, ws=ws)
    assert ws.nbytes > small
    others = [torch.full((small,), 7, dtype=torch.uint8, device="cuda") for _ in range(8)]
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and all(bool((t == 7).all()) for t in others)


@gpu
def test_an_outgrown_buffer_waits_for_the_streams_that_had_it():
    """A buffer made on one stream and given to a call on another: once outgrown, its memory goes to no tensor of the first
    stream before the second one's work has ended."""
    n = 32 << 20
    ws, s = bd.Workspace(), torch.cuda.Stream()
    at = ws.ensure(n).data_ptr()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        torch.cuda._sleep(int(2e8))  # some 0.1 s, in place of a long call
        ws.ensure(n)
        done = torch.cuda.Event()
        done.record()
        ws.ensure(2 * n)
    other = torch.empty(n, dtype=torch.uint8, device="cuda")
    assert not done.query(), "the stream was through before the tensor was made"
    assert other.data_ptr() != at
    torch.cuda.synchronize()
