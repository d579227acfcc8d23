"""The softmax attention layer on pages of a cache: prompts, prompts that go on, single tokens and drafts against float64.

Each of the eight tensors between its operators (the rounded weights of attention among them) is rounded to bf16 (2^-8 relative at
most).  None of the steps after it enlarges a relative error by more than two: scores are of the size of one, so an error of q
or k is one of the same size in the weights, and attention averages v and the weights' errors alike.  So results are within
8 * 2 * 2^-8 of the definition in the 2-norm.
"""
import numpy as np
import pytest
import torch

from oracle import seqmix as ref
from paper_2407_10730_amd.mixer import Pages, SoftmaxLayer, main
from test_gpu_mixer import TOL, _host, _off

pytestmark = pytest.mark.gpu
WIDTH = 256


def _layer(slots=5, page=16, pages=60, max_pages=20, **kw):
    pool = Pages(slots=slots, page=page, pages=pages, max_pages=max_pages)
    return pool, SoftmaxLayer(pool, width=WIDTH, heads=4, kv_heads=2, dim=64, **kw)


def _x(n, seed=0):
    return torch.randn(n, WIDTH, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)).bfloat16()


def _ints(*i):
    return torch.tensor(i, dtype=torch.int32, device="cuda")


def _offsets(lens):
    return torch.tensor([0] + list(lens), device="cuda").cumsum(0)


def _want(layer, x, see=None):
    """The layer's definition for one text; see: which rows each row sees (None: those up to itself)."""
    H, D, n = _host, layer, len(x)
    h, _ = ref.norm(H(x), "rms", H(D.n_in), None, 1e-6)
    q, k, v = (t.reshape(n, -1, D.dim) for t in np.split(h @ H(D.w_in).T, [D.inner, D.inner + D.kv_heads * D.dim], 1))
    f = D.freqs.cpu().numpy()
    pos = np.arange(n) if see is None else see[1]
    q, k = (ref.rotary(t, pos, f, D.dim, "half", 1.0) for t in (q, k))
    o, _, _ = ref.softmax_attention(q, k, v, np.tri(n, dtype=bool) if see is None else see[0], D.dim ** -0.5)
    u, _ = ref.norm(o.reshape(n, -1) @ H(D.w_out).T, "rms", H(D.n_out), None, 1e-6)
    y = H(x) + D.scale * u
    return y, ref.norm(y, "rms", H(D.n_next), None, 1e-6)[0]


def test_prompts_parts_and_tokens():
    pool, layer = _layer()
    lens = [100, 37, 1, 70]
    xs = [_x(n, i) for i, n in enumerate(lens)]
    want = [_want(layer, x) for x in xs]
    slots = _ints(4, 0, 2, 1)

    def near(got, rows):
        for i, (a, b) in enumerate(rows):
            for part, whole in zip(got, want[i]):
                if b > a:
                    first = sum(d - c for c, d in rows[:i])
                    assert _off(_host(part[first:first + b - a]), whole[a:b]) <= TOL

    def call(rows):
        off = _offsets([b - a for a, b in rows])
        x = torch.cat([x[a:b] for x, (a, b) in zip(xs, rows)])
        near(layer.run(x, pool.step(len(x), slots, off), off), rows)

    call([(0, n) for n in lens])
    pool.step(0, slots, _offsets([0] * 4), torch.zeros_like(slots))  # all end
    assert pool.taken.item() == 0 and not pool.lens.any()
    at = [60, 33, 0, 65]
    call([(0, n) for n in at])
    call([(a, max(a, n - 2)) for a, n in zip(at, lens)])
    at = [max(a, n - 2) for a, n in zip(at, lens)]
    while any(a < n for a, n in zip(at, lens)):
        call([(a, min(a + 1, n)) for a, n in zip(at, lens)])
        at = [min(a + 1, n) for a, n in zip(at, lens)]
    assert pool.lens[slots.long()].tolist() == lens


def test_drafts():
    """Drafted rows of two requests see their own branch; the branch that was kept goes on as a text without drafts would."""
    pool, layer = _layer()
    text, branch = [_x(40, 1), _x(9, 2)], _x(6, 3)
    slots = _ints(3, 1)
    off = _offsets([40, 9])
    layer.run(torch.cat(text), pool.step(49, slots, off), off)
    off = _offsets([3, 3])  # a chain of two, and another first token
    tree = torch.tensor([1, 3, 4], device="cuda").repeat(2)
    got = layer.run(branch, pool.step(6, slots, off), off, tree)
    for i, t in enumerate(text):
        n = len(t)
        see = np.tri(n + 3, dtype=bool)
        see[n + 2, n:n + 2] = False
        want = _want(layer, torch.cat([t, branch[3 * i:3 * i + 3]]), (see, np.arange(n + 3)))
        for g, w in zip(got, want):
            assert _off(_host(g[3 * i:3 * i + 3]), w[n:]) <= TOL
    # the chain is kept, the other goes
    more = _x(2, 4)
    got = layer.run(more, pool.step(2, slots, kept=_ints(42, 11)))
    for i, t in enumerate(text):
        want = _want(layer, torch.cat([t, branch[3 * i:3 * i + 2], more[i:i + 1]]))
        for g, w in zip(got, want):
            assert _off(_host(g[i:i + 1]), w[-1:]) <= TOL


def test_requests_without_room_pass_through():
    pool, layer = _layer(pages=7)
    layer.run(100 * _x(90, 7), pool.step(90, _ints(0, 1), _offsets([45, 45])), _offsets([45, 45]))  # another user's rows
    pool.step(0, _ints(0, 1), _offsets([0, 0]), _ints(0, 0))
    x, off = _x(95, 1), _offsets([40, 50, 5])  # 3, 4 and 1 pages of 7; the second's slot is outside the pool
    places = pool.step(95, _ints(2, 9, 0), off)
    assert places[2].tolist() == [2, -1, 0]
    y, h = layer.run(x, places, off)
    assert torch.equal(y[40:90], x[40:90])
    assert _off(_host(h[40:90]), ref.norm(_host(x[40:90]), "rms", _host(layer.n_next), None, 1e-6)[0]) <= TOL
    for rows in (slice(0, 40), slice(90, 95)):
        for got, want in zip((y, h), _want(layer, x[rows])):
            assert _off(_host(got[rows]), want) <= TOL
    full = pool.step(60, _ints(1), _offsets([60]))  # 4 pages where 3 are left
    assert full[2].tolist() == [-1] and torch.equal(layer.run(x[:60], full, _offsets([60]))[0], x[:60])


def test_sizes_come_and_go():
    pool, layer = _layer(plans=4)
    for n in range(1, 20):
        off = _offsets([n])
        places = pool.step(n, _ints(0), off, _ints(0))
        layer.run(_x(n), places, off)
    assert len(layer._plans) <= 4
    off = _offsets([7])
    got = layer.run(_x(7), pool.step(7, _ints(0), off, _ints(0)), off)
    for g, w in zip(got, _want(layer, _x(7))):
        assert _off(_host(g), w) <= TOL


def test_captured_steps():
    """A captured step of single tokens, replayed between other calls, is the eager one."""
    pool, layer = _layer()
    slots, x = _ints(2, 0, 1), _x(3)
    off = _offsets([50, 3, 17])
    layer.run(_x(70, 5), pool.step(70, slots, off), off)
    layer.run(x, pool.step(3, slots))
    state = (pool.lens, pool.table, pool.free, pool.taken, layer.k_cache, layer.v_cache)
    torch.cuda.synchronize()
    before = [t.clone() for t in state]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, h = layer.run(x, pool.step(3, slots))
    for t, b in zip(state, before):
        assert torch.equal(t, b)
    for i in range(4):
        other = _offsets([9 + i])
        layer.run(_x(9 + i), pool.step(9 + i, _ints(4), other, _ints(0)), other)
        x.copy_(_x(3, 20 + i))
        before = [t.clone() for t in state]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (y, h, *state)]
        for t, b in zip(state, before):
            t.copy_(b)
        want = layer.run(x, pool.step(3, slots))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (*want, *state)))


def test_the_command_times_it(capsys):
    main(["--requests", "3", "--prompt", "50", "--steps", "2"])
    assert "softmax attention, one token each" in capsys.readouterr().out
