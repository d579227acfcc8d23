"""Attention with a workspace under graph capture, beside eager calls on other streams (needs the GPU)."""
import pytest
import torch

from test_gpu_seqmix import Attn, _gpu  # noqa: F401

pytestmark = pytest.mark.gpu


def _eager(a, stream=None):
    left = torch.empty_like(a.state)
    a.run(a.state, left, stream=stream)
    torch.cuda.synchronize()
    return a.o.clone(), left


def _renew(a, seed):
    for i, t in enumerate((a.q, a.k, a.v, a.state)):
        t.normal_(generator=torch.Generator(device="cuda").manual_seed(10 * seed + i))
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_capture_after_calls_on_other_streams(dtype):
    """The capture's stream is a new one; eager calls, on two streams, come before it and between its replays."""
    a = Attn([900], 2, 2, 64, 64, dtype=dtype)
    assert a.op.plan().workspace_bytes > 0
    side = torch.cuda.Stream()
    _eager(a)
    left, graph = torch.empty_like(a.state), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.run(a.state, left)
    for i in range(4):
        _renew(a, i)
        graph.replay()
        torch.cuda.synchronize()
        got = a.o.clone(), left.clone()
        for want in (_eager(a), _eager(a, side)):
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_streams_of_one_capture_wait_for_each_other():
    """Two calls of a descriptor on two streams that the capture forks to, without an edge of the caller's between them."""
    a, b = Attn([4000], 2, 1, 64, 64, seed=1), Attn([4000], 2, 1, 64, 64, seed=2)
    want = [_eager(a), _eager(b)]
    a.op.reserve()
    lefts = [torch.empty_like(a.state) for _ in range(2)]
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph):
        here = torch.cuda.current_stream()
        side.wait_stream(here)
        for x, s, left in ((a, here, lefts[0]), (b, side, lefts[1])):
            a.op.run(x.q, x.k, x.v, x.g, x.state, left, x.o, stream=s)
        here.wait_stream(side)
    for _ in range(4):
        for t in (a.o, b.o, *lefts):
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for x, left, (o, state) in zip((a, b), lefts, want):
            assert torch.equal(x.o, o) and torch.equal(left, state)
        _eager(a)


def test_two_captures_of_one_descriptor():
    a = Attn([900], 2, 2, 64, 64)
    _eager(a)
    left, graphs = torch.empty_like(a.state), [torch.cuda.CUDAGraph() for _ in range(2)]
    for g in graphs:
        with torch.cuda.graph(g):
            a.run(a.state, left)
    for i in range(3):
        for g in graphs:
            _renew(a, i)
            g.replay()
            torch.cuda.synchronize()
            got = a.o.clone(), left.clone()
            want = _eager(a)
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_eager_call_during_a_capture_is_no_part_of_it():
    """Between two captured calls, on a stream of its own: it runs at once, and the graph holds the others alone."""
    a, b = Attn([900], 2, 2, 64, 64, seed=1), Attn([900], 2, 2, 64, 64, seed=2)
    (o_a, state_a), (o_b, state_b) = _eager(a), _eager(b)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    lefts = [torch.zeros_like(a.state) for _ in range(2)]
    a.op.reserve()
    for t in (a.o, b.o):
        t.zero_()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        a.run(a.state, lefts[0])
        a.op.run(b.q, b.k, b.v, b.g, b.state, lefts[1], b.o, stream=side)
        a.run(a.state, lefts[0])
    torch.cuda.synchronize()
    assert torch.equal(b.o, o_b) and torch.equal(lefts[1], state_b) and not a.o.any()
    for _ in range(3):
        for t in (a.o, b.o, *lefts):
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(a.o, o_a) and torch.equal(lefts[0], state_a) and not b.o.any() and not lefts[1].any()
