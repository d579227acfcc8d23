"""The gated linear-attention layer as a serving program uses it: many sizes, several streams, empty places, graphs (needs the GPU)."""
import pytest
import torch

from oracle import seqmix as ref
from paper_2407_10730_amd.mixer import MixerLayer
from test_gpu_mixer import TOL, _host, _off

pytestmark = pytest.mark.gpu


def _layer(**kw):
    return MixerLayer(width=256, heads=4, qk_heads=2, dk=64, dv=64, slots=6, **kw)


def _x(n, seed=0):
    return torch.randn(n, 256, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)).bfloat16()


def _slots(*i):
    return torch.tensor(i, dtype=torch.int32, device="cuda")


def test_many_sizes_keep_little():
    """Sizes that come once leave neither buffers nor, past the bound, descriptors behind."""
    layer = _layer(plans=4)
    slots = _slots(0)
    layer.run(_x(40), slots)
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    for n in range(100, 130):
        layer.clear(slots)
        layer.run(_x(n), slots)
    torch.cuda.synchronize()
    assert torch.cuda.memory_allocated() <= before + (1 << 20)  # a call's tensors are 0.6 MB
    assert len(layer._plans) <= 4
    layer.clear(slots)  # a size whose descriptors went computes the same
    first = [t.clone() for t in layer.run(_x(129), slots)]
    for n in range(60, 70):
        layer.run(_x(n), slots)
    layer.clear(slots)
    again = layer.run(_x(129), slots)
    assert all(torch.equal(a, b) for a, b in zip(first, again))


@pytest.mark.parametrize("n", [1, 700])
def test_streams_with_slots_of_their_own(n):
    """Calls of one size, side by side on two streams, do not meet in a buffer."""
    layer = _layer()
    xs, slots = [_x(3 * n, 1), _x(3 * n, 2)], [_slots(0, 1, 2), _slots(5, 4, 3)]
    want = []
    for x, i in zip(xs, slots):
        want.append([t.clone() for t in layer.run(x, i)])
    states = layer.states.clone()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        layer.clear(torch.cat(slots))
        torch.cuda.synchronize()
        got = []
        for x, i, s in zip(xs, slots, streams):
            with torch.cuda.stream(s):
                got.append(layer.run(x, i))
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            assert torch.equal(g[0], w[0]) and torch.equal(g[1], w[1])
        assert torch.equal(layer.states, states)


@pytest.mark.parametrize("lens", [[1, 1, 1], [40, 3, 25]])
def test_empty_places_pass_through(lens):
    """A request without a slot: x' is x, whatever ran before, and nothing of the pool moves."""
    layer = _layer()
    n = sum(lens)
    offsets = None if lens == [1, 1, 1] else torch.tensor([0] + lens, device="cuda").cumsum(0)
    layer.run(100 * _x(n, 7), _slots(0, 1, 2), offsets)  # another user's rows in memory of these sizes
    layer.clear(_slots(0, 1, 2))
    before = layer.states.clone(), layer.windows.clone()
    x = _x(n)
    y, h = layer.run(x, _slots(0, -1, 6), offsets)
    rows = slice(lens[0], n)
    assert torch.equal(y[rows], x[rows])
    want, _ = ref.norm(_host(x[rows]), "rms", _host(layer.n_next), None, 1e-6)
    assert _off(_host(h[rows]), want) <= TOL
    assert torch.equal(layer.states[1:], before[0][1:]) and torch.equal(layer.windows[1:], before[1][1:])
    alone, alone_h = (t.clone() for t in layer.run(x[:lens[0]].contiguous(), _slots(3)))
    assert _off(_host(y[:lens[0]]), _host(alone)) <= TOL and _off(_host(h[:lens[0]]), _host(alone_h)) <= TOL


def test_graph_keeps_its_descriptors():
    """A captured decoding step runs right after many other sizes have come and gone."""
    layer = _layer(plans=2)
    slots, x = _slots(2, 0, 1), _x(3)
    layer.run(x, slots)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, h = layer.run(x, slots)
    for i in range(3):
        for n in (5, 90 + i, 200 + i, 300 + i):
            layer.run(_x(n), _slots(5))
        states, windows = layer.states.clone(), layer.windows.clone()
        x.copy_(_x(3, 20 + i))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = y.clone(), h.clone(), layer.states.clone()
        layer.states.copy_(states)
        layer.windows.copy_(windows)
        want = layer.run(x, slots)
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and torch.equal(got[2], layer.states)
