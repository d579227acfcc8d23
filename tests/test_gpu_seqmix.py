"""Token-mixing operators against their float64 definitions (needs the GPU).

Errors are taken relative to the same sums over absolute values (`oracle.seqmix`), point by point.
With u = 2^-24 (fp32) and r = 2^-8 (one rounding to bf16: 8 significant bits, half a unit in the last of them):

 * attention, fp32: a term passes through at most 2 roundings per token of the sequence (decay and
   sum), one per chunk or key column summed, and an exponential whose argument is rounded: (2 T + dk + 64) u.
   bf16 outputs: scores and states enter the matrix product rounded to bf16 once each, and the output is
   rounded once: 2 r more.  States keep the fp32 bound for either type.
 * convolution: W products and sums and the bias, (W + 2) u; SiLU has a slope below 1.1 and its own
   error of (|z| + 8) u |y|; bf16 rounds once: r |y|.
 * norm: sums of at most 64 values in a row in one thread, then 10 levels of pairs and 16 waves:
   96 u for each mean, twice with LAYER; the gate's sigmoid (|z| + 8) u; the second norm adds its own and
   passes the first one's on.  bf16 rounds once: r.
"""
import numpy as np
import pytest
import torch

from oracle import seqmix as ref
from paper_2407_10730_amd import binding as B
from paper_2407_10730_amd import seqmix as M

pytestmark = pytest.mark.gpu

U, R = 2.0 ** -24, 2.0 ** -8
TD = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    M.load()
    yield
    torch.cuda.synchronize()


def _host(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def _near(got, want, size, tol, what):
    """Point by point within tol * size; infinite and NaN where the definition is."""
    fine = np.isfinite(want)
    assert np.array_equal(np.isfinite(got), fine), f"{what}: finite in other places"
    err = np.abs(got - want)[fine]
    bound = (tol * size + 1e-37)[fine] if np.ndim(tol) else tol * size[fine] + 1e-37
    if err.size:
        worst = float((err / bound).max())
        print(f"  {what}: {worst:.3f} of the bound", flush=True)
        assert worst <= 1.0, f"{what}: {worst:.3g} times the bound"


class Attn:
    """One attention problem on the GPU, its tensors strided or shifted as asked, and its definition."""

    def __init__(self, lens, heads, qk_heads, dk, dv, dtype="bf16", decay="token", o_dtype=None, seed=0, shift=0, pad=0,
                 heads_outer=False, uniform=None, state=True, pool=0, scale=0.37, edit=None):
        rng = np.random.default_rng(seed)
        self.lens, self.n = lens, sum(lens)
        n, td = self.n, TD[dtype]
        self.dtype, self.heads, self.dk, self.dv, self.scale = dtype, heads, dk, dv, scale

        def dev(h, d, t=td):  # a strided home for [n, h, d]
            if heads_outer:
                flat = torch.zeros(h * (n + 1) * (d + pad) + shift + 16, dtype=t, device="cuda")
                return flat[shift:].as_strided((n, h, d), (d + pad, (n + 1) * (d + pad), 1))
            flat = torch.zeros((n + 1) * (h * d + pad) + shift + 16, dtype=t, device="cuda")
            return flat[shift:].as_strided((n, h, d), (h * d + pad, d, 1))

        self.q, self.k, self.v = dev(qk_heads, dk), dev(qk_heads, dk), dev(heads, dv)
        self.o = dev(heads, dv, TD[o_dtype or dtype])
        for t, s in ((self.q, 1.0), (self.k, dk ** -0.5), (self.v, 1.0)):
            t.copy_(torch.from_numpy(rng.standard_normal(tuple(t.shape)) * s).to(td))
        if decay == "token":
            g = -np.exp(rng.standard_normal((n, heads)) * 1.5 - 3)
        else:
            g = -np.exp(rng.standard_normal(heads) - 3) if decay == "head" else None
        self.g = None if g is None else torch.from_numpy(g).float().cuda()
        if edit:
            edit(self)
        self.slots = len(lens) + pool
        self.index = rng.permutation(self.slots)[:len(lens)] if pool else np.arange(len(lens))
        self.slot_t = torch.from_numpy(self.index.astype(np.int32)).cuda() if pool else None
        self.state = torch.from_numpy(rng.standard_normal((self.slots, heads, dk, dv))).float().cuda() if state else None
        uniform = len(set(lens)) == 1 if uniform is None else uniform
        self.off_t = None if uniform else torch.tensor([0] + lens, device="cuda").cumsum(0)
        self.op = M.LinearAttention(
            tokens=n, seqs=len(lens), slots=self.slots, heads=heads, qk_heads=qk_heads, dk=dk, dv=dv, dtype=dtype,
            o_dtype=o_dtype, decay=decay, scale=scale, q_strides=self.q.stride()[:2], k_strides=self.k.stride()[:2],
            v_strides=self.v.stride()[:2], o_strides=self.o.stride()[:2])

    def run(self, state_in, state_out, **kw):
        self.op.run(self.q, self.k, self.v, self.g, state_in, state_out, self.o, offsets=self.off_t,
                    slot_index=self.slot_t, **kw)
        return self

    def want(self):
        g = np.zeros((self.n, self.heads))
        if self.g is not None:
            g = np.broadcast_to(_host(self.g), g.shape)
        first = _host(self.state)[self.index] if self.state is not None else np.zeros(
            (len(self.lens), self.heads, self.dk, self.dv))
        return ref.linear_attention(_host(self.q), _host(self.k), _host(self.v), g, self.lens, first, self.scale)

    def check(self, left=None):
        o, o_abs, s, s_abs = self.want()
        f32 = (2 * max(self.lens + [1]) + self.dk + 64) * U
        half = 0 if self.dtype == "f32" else 2 * R
        _near(_host(self.o), o, o_abs, f32 + half, "o")
        if left is not None:
            _near(_host(left)[self.index], s, s_abs, f32, "state")


def _case(**kw):
    return pytest.param(kw, id="-".join(f"{k}{v}" for k, v in kw.items()).replace(" ", ""))


ATTN = [
    # single tokens: head sizes that fill tiles and that do not, shared heads
    _case(lens=[1] * 3, heads=4, qk_heads=2, dk=128, dv=128),
    _case(lens=[1] * 3, heads=4, qk_heads=4, dk=64, dv=64, dtype="f32", decay="head"),
    _case(lens=[1], heads=1, qk_heads=1, dk=1, dv=1),
    _case(lens=[1] * 2, heads=3, qk_heads=1, dk=33, dv=70, dtype="f32", decay="none"),
    _case(lens=[1] * 2, heads=2, qk_heads=1, dk=256, dv=256, o_dtype="f32"),
    _case(lens=[1] * 2, heads=2, qk_heads=2, dk=200, dv=36),
    # a few tokens
    _case(lens=[5] * 4, heads=2, qk_heads=1, dk=96, dv=128),
    # around the edges of chunks and segments
    *[_case(lens=[t], heads=2, qk_heads=1, dk=64, dv=64) for t in (15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129)],
    *[_case(lens=[t], heads=2, qk_heads=1, dk=32, dv=48, dtype="f32") for t in (15, 16, 17, 31, 33, 63, 64, 65, 129)],
    _case(lens=[300], heads=2, qk_heads=2, dk=128, dv=128, decay="head"),
    _case(lens=[300], heads=2, qk_heads=2, dk=128, dv=128, decay="none", o_dtype="f32"),
    _case(lens=[260], heads=1, qk_heads=1, dk=256, dv=256),
    _case(lens=[260], heads=1, qk_heads=1, dk=256, dv=256, dtype="f32"),
    _case(lens=[260], heads=1, qk_heads=1, dk=200, dv=132),
    _case(lens=[260], heads=1, qk_heads=1, dk=72, dv=40, dtype="f32", decay="head"),
    _case(lens=[130], heads=2, qk_heads=1, dk=33, dv=71),
    _case(lens=[130], heads=2, qk_heads=1, dk=17, dv=9, dtype="f32"),
    _case(lens=[700], heads=1, qk_heads=1, dk=16, dv=16),
    _case(lens=[700], heads=1, qk_heads=1, dk=16, dv=16, dtype="f32"),
    # ragged, with empty sequences at every place
    _case(lens=[0, 70, 1, 0, 0, 200, 64, 3, 0], heads=3, qk_heads=1, dk=64, dv=96),
    _case(lens=[0, 70, 1, 0, 0, 200, 64, 3, 0], heads=2, qk_heads=2, dk=40, dv=128, dtype="f32"),
    _case(lens=[1, 0, 2, 1, 1], heads=2, qk_heads=2, dk=128, dv=64),
    _case(lens=[90] * 5, heads=2, qk_heads=1, dk=128, dv=128),
    _case(lens=[90] * 5, heads=2, qk_heads=1, dk=128, dv=128, uniform=False),
]


@pytest.mark.parametrize("kw", ATTN)
@pytest.mark.parametrize("carry", ["pool", "zero"])
def test_attention(kw, carry):
    print(f"\n[case] {kw} {carry}", flush=True)
    if carry == "zero":  # starts from nothing, keeps what is left apart
        a = Attn(**kw, state=False)
        left = torch.full((a.slots, a.heads, a.dk, a.dv), 7.0, device="cuda")
        a.run(None, left).check(left)
        return
    a = Attn(**kw, pool=2)  # in place in a pool, whose other entries stay
    left, other = a.state.clone(), np.setdiff1d(np.arange(a.slots), a.index)
    a.run(left, left).check(left)
    assert torch.equal(left[other], a.state[other])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_many_sequences(dtype):
    """More sequences than a wave looks up at once, and than one step of its search covers; some of them cut."""
    rng = np.random.default_rng(2)
    lens = [int(t) for t in rng.integers(0, 12, 150)]
    lens[70] = 400
    a = Attn(lens, 1, 1, 32, 32, dtype=dtype, uniform=False, pool=4)
    left = a.state.clone()
    a.run(left, left).check(left)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens,uniform", [([2000], None), ([900, 900], None), ([1500, 0, 800, 1], False)])
def test_attention_in_segments(dtype, lens, uniform):
    """Long enough to be cut, also where the last segment is short."""
    a = Attn(lens, 2, 2, 64, 96, dtype=dtype, uniform=uniform)
    plan = a.op.plan()
    assert plan.kernel == M.SEQMIX_KERNEL_CHUNKS and 0 < plan.segment < max(lens) and plan.workspace_bytes > 0
    left = torch.empty_like(a.state)
    a.run(a.state, left).check(left)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,qk_heads", [(2, 1), (16, 16)])
@pytest.mark.parametrize("lens", [[1] * 64 + [1000], [1] * 20 + [700, 0, 0, 650] + [1] * 30 + [129], [570, 1, 3],
                                  [64, 65, 96, 97, 127, 128, 129, 130, 191, 192, 193, 300]], ids=lambda x: f"{len(x)}-{sum(x)}")
def test_attention_some_cut(dtype, heads, qk_heads, lens):
    """Packs of which the long sequences are cut and the others are not, in place in a pool."""
    a = Attn(lens, heads, qk_heads, 64, 72, dtype=dtype, pool=3, uniform=False)
    plan = a.op.plan()
    assert plan.kernel == M.SEQMIX_KERNEL_CHUNKS and 0 < plan.segment < max(lens)
    left, other = a.state.clone(), np.setdiff1d(np.arange(a.slots), a.index)
    a.run(left, left).check(left)
    assert torch.equal(left[other], a.state[other])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens", [[3], [100]])
def test_attention_growing_decays(dtype, lens):
    """Log decays above 0, growing by far more than a chunk's terms are of."""
    def edit(a):
        a.g.uniform_(-0.2, 0.6, generator=torch.Generator(device="cuda").manual_seed(1))

    a = Attn(lens, 2, 2, 64, 64, dtype=dtype, edit=edit)
    left = torch.empty_like(a.state)
    a.run(a.state, left).check(left)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens", [[1, 1], [150, 40]])
@pytest.mark.parametrize("kw", [dict(shift=1), dict(pad=24), dict(pad=3), dict(heads_outer=True),
                                dict(heads_outer=True, shift=3, pad=1)], ids=str)
def test_attention_strides(dtype, lens, kw):
    a = Attn(lens, 4, 2, 64, 128, dtype=dtype, uniform=False, **kw)
    left = torch.empty_like(a.state)
    a.run(a.state, left).check(left)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens", [[1] * 2, [3] * 160, [150, 0, 40], [700]], ids=["1x2", "3x160", "150,0,40", "700"])
@pytest.mark.parametrize("dk,dv", [(9, 8), (8, 13), (3, 5), (7, 130), (131, 2), (15, 129), (127, 3), (250, 67), (2, 1),
                                   (36, 189), (68, 98)])
def test_attention_odd_heads_between_nan(dtype, lens, dk, dv):
    """Rows end inside a load, and what lies beside them is no operand and stays as it is."""
    def edit(a):
        for t in (a.q, a.k, a.v):
            keep = t.clone()
            t._base.fill_(float("nan"))
            t.copy_(keep)
        a.o._base.fill_(5.0)

    a = Attn(lens, 2, 1, dk, dv, dtype=dtype, pad=3, shift=1, edit=edit, uniform=False)
    left = torch.full((a.slots + 1, a.heads, dk, dv), 3.0, device="cuda")
    a.run(a.state, left[:-1]).check(left[:-1])
    a.o.fill_(5.0)
    assert bool((a.o._base == 5.0).all()) and bool((left[-1] == 3.0).all())
    left[:-1] = a.state  # in place
    a.run(left[:-1], left[:-1]).check(left[:-1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens", [[1, 1, 1], [4, 4, 4], [150, 70, 0], [700]])
def test_attention_decays_that_clear_the_state(dtype, lens):
    """-infinity (and the type's lowest value) as the log of a decay, also many of them and of other sizes between."""
    def edit(a):
        rng = np.random.default_rng(3)
        at = torch.from_numpy(rng.random(tuple(a.g.shape)) < 0.15).cuda()
        a.g[at] = -float("inf")
        a.g[torch.from_numpy(rng.random(tuple(a.g.shape)) < 0.05).cuda()] = torch.finfo(torch.float32).min
        a.g[torch.from_numpy(rng.random(tuple(a.g.shape)) < 0.1).cuda()] = -150.0

    a = Attn(lens, 3, 3, 48, 64, dtype=dtype, edit=edit, uniform=False)
    left = torch.empty_like(a.state)
    a.run(a.state, left).check(left)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("where", ["q", "k", "v", "g"])
@pytest.mark.parametrize("value", [float("inf"), float("nan")])
@pytest.mark.parametrize("at", [0, 7, 45, 99])
def test_attention_keeps_the_past_from_the_future(dtype, where, value, at):
    """Outputs before a token with an infinite or NaN value are what they are without it, and so is another sequence."""
    bad = Attn([100, 60], 2, 1, 64, 64, dtype=dtype, seed=5)
    good = Attn([100, 60], 2, 1, 64, 64, dtype=dtype, seed=5)
    if where == "g":
        bad.g[at, :] = value
    else:
        t = getattr(bad, where)
        t[at, :, 3] = value
    left = torch.empty_like(bad.state)
    bad.run(bad.state, left)
    good.run(good.state, torch.empty_like(left))
    got, want = _host(bad.o), _host(good.o)
    r = 2 * R if dtype == "bf16" else 0  # a bound, as the two may sum in another order
    _, o_abs, _, _ = good.want()
    f32 = (2 * 100 + 64 + 64) * U
    for rows in (slice(0, at), slice(100, 160)):
        _near(got[rows], want[rows], o_abs[rows], 2 * (f32 + r), "rows apart")
    assert not np.isfinite(got[at]).all()  # q and v: its own column or row; k, g: all that follows
    if where == "q":
        _near(got[at + 1:100], want[at + 1:100], o_abs[at + 1:100], 2 * (f32 + r), "rows after")
    if where == "v":  # one column of it and of what follows
        keep = [c for c in range(64) if c != 3]
        _near(got[:, :, keep], want[:, :, keep], o_abs[:, :, keep], 2 * (f32 + r), "other columns")
        assert not np.isfinite(got[at:100, :, 3]).any()
        assert np.isfinite(_host(left)[0][:, :, keep]).all() and not np.isfinite(_host(left)[0][:, :, 3]).any()


def test_attention_skips_empty_places():
    for lens in ([1] * 4, [70, 1, 90, 30]):
        a = Attn(lens, 2, 2, 64, 64, pool=3, uniform=False)
        left = a.state.clone()
        index = a.slot_t.clone()
        a.slot_t[1], a.slot_t[3] = -1, a.slots  # skipped
        a.o.fill_(5.0)
        a.run(left, left)
        o, o_abs, s, s_abs = a.want()
        first = np.cumsum([0] + lens)
        for i in range(4):
            rows = slice(first[i], first[i + 1])
            slot = int(index[i])
            if i in (1, 3):
                assert bool((a.o[rows] == 5.0).all()) and torch.equal(left[slot], a.state[slot])
            else:
                _near(_host(a.o)[rows], o[rows], o_abs[rows], 2 * R + 400 * U, "o")
                _near(_host(left)[slot], s[i], s_abs[i], 400 * U, "state")


def test_attention_without_tokens():
    a = Attn([0, 0], 2, 1, 16, 16)
    left = torch.full_like(a.state, 9.0)
    a.run(a.state, left)
    assert torch.equal(left, a.state)
    a.run(None, left)
    assert not left.any()


def test_attention_offsets_out_of_range_stay_inside():
    """Offsets that lie give wrong results, not accesses outside the tensors."""
    a = Attn([100, 28], 1, 1, 32, 32, uniform=False)
    left = torch.empty_like(a.state)
    for off in ([0, 1 << 40, 128], [-50, 500, 128], [90, 20, 10], [-(1 << 50), -5, -1], [1 << 50, 1 << 51, 1 << 52]):
        a.off_t = torch.tensor(off, device="cuda")
        a.run(a.state, left)
        torch.cuda.synchronize()


@pytest.mark.parametrize("lens", [[70], [3]])
def test_attention_rows_past_32_bits(lens):
    """Rows 2^26 elements apart: offsets pass 2^31 elements."""
    n, row = lens[0], (1 << 26) + 8
    if n == 3:
        row = (1 << 30) + 8
    a = Attn(lens, 2, 2, 64, 64)
    far = torch.empty((n - 1) * row + 128, dtype=torch.bfloat16, device="cuda")
    view = far.as_strided((n, 2, 64), (row, 64, 1))
    view.copy_(a.q)
    o = torch.empty(n, 2, 64, dtype=torch.bfloat16, device="cuda")
    op = M.LinearAttention(tokens=n, seqs=1, heads=2, dk=64, dv=64, scale=a.scale, q_strides=(row, 64))
    left = torch.empty_like(a.state)
    op.run(view, a.k, a.v, a.g, a.state, left, o)
    a.o.copy_(o)
    a.check(left)
    op = M.LinearAttention(tokens=n, seqs=1, heads=2, dk=64, dv=64, scale=a.scale, v_strides=(row, 64),
                           o_strides=(row, 64))
    view.copy_(a.v)
    out = torch.empty((n - 1) * row + 128, dtype=torch.bfloat16, device="cuda").as_strided((n, 2, 64), (row, 64, 1))
    op.run(a.q, a.k, view, a.g, a.state, left, out)
    a.o.copy_(out)
    a.check(left)


def test_attention_on_streams():
    """One descriptor used on two streams in turn: the second call waits for the first one's workspace."""
    a = Attn([4000], 2, 1, 64, 64, seed=1)
    b = Attn([4000], 2, 1, 64, 64, seed=2)
    want = []
    for x in (a, b):
        left = torch.empty_like(x.state)
        x.run(x.state, left)
        want.append((x.o.clone(), left))
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(4):
        lefts = [torch.zeros_like(a.state) for _ in range(2)]
        a.o.zero_()
        b.o.zero_()
        torch.cuda.synchronize()
        for x, s, left in ((a, s1, lefts[0]), (b, s2, lefts[1])):
            a.op.run(x.q, x.k, x.v, x.g, x.state, left, x.o, stream=s)
        torch.cuda.synchronize()
        for x, (o, left), got in zip((a, b), want, lefts):
            assert torch.equal(x.o, o) and torch.equal(got, left)


@pytest.mark.parametrize("lens", [[1] * 4, [900]])
def test_operators_in_a_graph(lens):
    """Captured once, replayed on other inputs with eager work between."""
    n, h, d = sum(lens), 2, 64
    a = Attn(lens, h, h, d, d, pool=1)
    a.op.reserve()
    rows = a.op.params.tokens
    conv = M.TokenConv(tokens=n, seqs=len(lens), slots=a.slots, channels=h * d, width=4)
    norm = M.GateNorm(rows=rows, width=h * d, group=d, gate="silu")
    w, bias, pw = torch.randn(h * d, 4, device="cuda").bfloat16(), torch.randn(h * d, device="cuda"), torch.rand(
        d, device="cuda")
    x, y = torch.randn(n, h * d, device="cuda").bfloat16(), torch.empty(n, h * d, device="cuda").bfloat16()
    win = torch.zeros(a.slots, 3, h * d, device="cuda").bfloat16()
    v = torch.empty(n, h, d, device="cuda").bfloat16()
    state = a.state.clone()

    def step():
        conv.run(x, w, bias, win, win, v.view(n, h * d), slot_index=a.slot_t)
        a.op.run(a.q, a.k, v, a.g, state, state, a.o, slot_index=a.slot_t)
        norm.run(a.o.view(n, h * d), pw, gate=x, y=y)

    if a.o.stride() != v.stride():
        pytest.fail("the test's outputs are dense")
    step()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        step()  # the descriptor's last stream is the capture's
        s.synchronize()
        with torch.cuda.graph(graph, stream=s):
            step()
    torch.cuda.synchronize()
    for _ in range(3):
        x.normal_()
        win.normal_()
        before = (win.clone(), state.normal_().clone())
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (y, win, state)]
        win.copy_(before[0])
        state.copy_(before[1])
        with torch.cuda.stream(s):
            step()
        torch.cuda.synchronize()
        for g, e in zip(got, (y, win, state)):
            assert torch.equal(g, e)


CONV = [
    *[_case(lens=[1] * 3, channels=64, width=w) for w in (1, 2, 3, 4, 8)],
    *[_case(lens=[t], channels=40, width=4) for t in (1, 2, 3, 4, 5, 31, 32, 33, 64, 65, 100)],
    _case(lens=[70], channels=37, width=4),
    _case(lens=[70], channels=1, width=2, dtype="f32"),
    _case(lens=[70], channels=300, width=8, dtype="f32"),
    _case(lens=[0, 1, 2, 0, 3, 40, 0, 97], channels=72, width=4),
    _case(lens=[0, 1, 2, 0, 3, 40, 0, 97], channels=33, width=8, dtype="f32", act="none"),
    _case(lens=[9, 5, 1, 0], channels=2056, width=3, act="none", bias=False),
    _case(lens=[130], channels=5000, width=5, dtype="f32", bias=False),
    _case(lens=[33, 64], channels=64, width=4, pad=8),
    _case(lens=[33, 64], channels=64, width=4, pad=5, shift=1),
]


@pytest.mark.parametrize("kw", CONV)
@pytest.mark.parametrize("carry", ["in place", "apart", "zero"])
def test_token_conv(kw, carry):
    kw = dict(kw)
    print(f"\n[case] {kw} {carry}", flush=True)
    lens, c, width = kw["lens"], kw["channels"], kw["width"]
    dtype, act, bias = kw.get("dtype", "bf16"), kw.get("act", "silu"), kw.get("bias", True)
    pad, shift = kw.get("pad", 0), kw.get("shift", 0)
    n, td, rng = sum(lens), TD[dtype], np.random.default_rng(11)

    def home():
        return torch.zeros((n + 1) * (c + pad) + shift + 8, dtype=td, device="cuda")[shift:].as_strided((n, c), (c + pad, 1))

    x, y = home(), home()
    x.copy_(torch.from_numpy(rng.standard_normal((n, c))).to(td))
    w = torch.from_numpy(rng.standard_normal((c, width))).to(td).cuda()
    b = torch.from_numpy(rng.standard_normal(c)).float().cuda() if bias else None
    slots = len(lens) + 2
    index = rng.permutation(slots)[:len(lens)]
    pool = torch.from_numpy(rng.standard_normal((slots, width - 1, c))).to(td).cuda()
    op = M.TokenConv(tokens=n, seqs=len(lens), slots=slots, channels=c, width=width, dtype=dtype, act=act, bias=bias,
                     x_row=c + pad, y_row=c + pad)
    off = torch.tensor([0] + lens, device="cuda").cumsum(0) if len(set(lens)) > 1 else None
    slot_t = torch.from_numpy(index.astype(np.int32)).cuda()
    before = torch.zeros_like(pool) if carry == "zero" else pool
    out = pool.clone() if carry == "in place" else torch.full_like(pool, 3.0)
    op.run(x, w, b, None if carry == "zero" else out if carry == "in place" else pool, out, y, offsets=off,
           slot_index=slot_t)
    want, size, left = ref.token_conv(_host(x), _host(w), _host(b) if bias else 0.0, lens, _host(before)[index], act)
    z, _, _ = ref.token_conv(_host(x), _host(w), _host(b) if bias else 0.0, lens, _host(before)[index], "none")
    bound = 1.1 * (width + 2) * U * size + (np.abs(z) + 8) * U * np.abs(want) * (act == "silu")
    bound = bound * (1 + R) + (R * np.abs(want) if dtype == "bf16" else 0)
    _near(_host(y), want, bound, 1.0, "y")
    assert np.array_equal(_host(out)[index], left)  # copies
    other = np.setdiff1d(np.arange(slots), index)
    assert torch.equal(out[other], pool[other] if carry == "in place" else torch.full_like(pool[other], 3.0))


@pytest.mark.parametrize("kw", [_case(lens=[t], channels=c, width=4, dtype=d)
                                for t in (1, 45) for c in (5, 9, 2049, 2055) for d in ("bf16", "f32")])
@pytest.mark.parametrize("carry", ["in place", "zero"])
def test_token_conv_odd_channels(kw, carry):
    test_token_conv(kw, carry)


def test_token_conv_keeps_sequences_apart():
    """Infinities and NaN in one sequence and in skipped places reach no other sequence and no earlier token."""
    lens, c = [40, 40, 40], 64
    x = torch.randn(120, c, device="cuda").bfloat16()
    w, b = torch.randn(c, 4, device="cuda").bfloat16(), torch.zeros(c, device="cuda")
    op = M.TokenConv(tokens=120, seqs=3, channels=c, width=4)
    pool = torch.randn(3, 3, c, device="cuda").bfloat16()
    y, left = torch.empty_like(x), torch.empty_like(pool)
    op.run(x, w, b, pool, left, y)
    bad = x.clone()
    bad[45], bad[79] = float("nan"), float("inf")
    y2, left2 = torch.full_like(x, 4.0), torch.empty_like(pool)
    op.run(bad, w, b, pool, left2, y2)
    keep = [i for i in range(120) if not 45 <= i <= 48 and i != 79]
    assert torch.equal(y[keep], y2[keep]) and not torch.isfinite(y2[45:49].float()).any()
    assert torch.equal(left[[0, 2]], left2[[0, 2]])
    y2.fill_(4.0)
    op.run(x, w, b, pool, left2, y2, slot_index=torch.tensor([2, -1, 1], dtype=torch.int32, device="cuda"))
    assert bool((y2[40:80] == 4.0).all())


def test_token_conv_many_sequences():
    """More sequences than two steps of a wave's search cover."""
    rng = np.random.default_rng(4)
    lens = [int(t) for t in rng.integers(0, 3, 5000)]
    c = 40
    x = torch.randn(sum(lens), c, device="cuda")
    w = torch.randn(c, 3, device="cuda")
    pool = torch.randn(5000, 2, c, device="cuda")
    y, left = torch.empty_like(x), pool.clone()
    op = M.TokenConv(tokens=len(x), seqs=5000, channels=c, width=3, dtype="f32", bias=False, act="none")
    op.run(x, w, None, left, left, y, offsets=torch.tensor([0] + lens, device="cuda").cumsum(0))
    want, size, after = ref.token_conv(_host(x), _host(w), 0.0, lens, _host(pool), "none")
    _near(_host(y), want, 5 * U * size, 1.0, "y")
    assert np.array_equal(_host(left), after)


def test_token_conv_rows_past_32_bits():
    n, c, row = 40, 64, (1 << 26) + 8
    far = torch.empty((n - 1) * row + c, dtype=torch.bfloat16, device="cuda")
    x, near = far.as_strided((n, c), (row, 1)), torch.randn(n, c, device="cuda").bfloat16()
    x.copy_(near)
    w, y, y2 = torch.randn(c, 4, device="cuda").bfloat16(), torch.empty_like(near), torch.empty_like(near)
    left, left2 = (torch.empty(1, 3, c, device="cuda").bfloat16() for _ in range(2))
    M.TokenConv(tokens=n, seqs=1, channels=c, width=4, bias=False, x_row=row).run(x, w, None, None, left, y)
    M.TokenConv(tokens=n, seqs=1, channels=c, width=4, bias=False).run(near, w, None, None, left2, y2)
    assert torch.equal(y, y2) and torch.equal(left, left2)


NORM = [
    # widths from one element to the largest, of either load
    *[_case(rows=3, width=d) for d in (1, 8, 64, 120, 128, 130, 512, 1000, 1537, 2048, 4096, 8192, 12000, 16384)],
    *[_case(rows=3, width=d, dtype="f32", post="layer", pre="layer", residual=True)
      for d in (1, 4, 63, 64, 256, 257, 1024, 1030, 4096, 5000, 16380, 16383, 16384)],
    _case(rows=1, width=2048, gate="silu", residual=True, pre="rms"),
    _case(rows=700, width=1024, group=128, gate="silu"),
    _case(rows=13, width=1040, group=104, gate="silu", gate_first=True),
    _case(rows=13, width=15, group=5, gate="linear", dtype="f32"),
    _case(rows=37, width=768, gate="sigmoid", gate_run=10, residual=True, pre="layer", scale_vec=True, scale=-0.3),
    _case(rows=37, width=769, gate="sigmoid", gate_run=10, residual=True, pre="rms", scale_vec=True, res_dtype="f32"),
    _case(rows=37, width=640, residual=True, pre="rms", res_dtype="f32", gate="silu", gate_first=True),
    _case(rows=5, width=96, post="none", residual=True, pre="rms"),
    _case(rows=5, width=96, post="none", pre="layer", dtype="f32", no_y=True),
    _case(rows=5, width=500, post="none", gate="silu"),
    _case(rows=9, width=512, residual=True, pre="rms", pad=8),
    _case(rows=9, width=512, residual=True, pre="rms", pad=3, shift=1, gate="silu"),
    _case(rows=9, width=512, residual=True, pre="rms", alias=True),
    _case(rows=0, width=512, residual=True, pre="rms"),
]


@pytest.mark.parametrize("kw", NORM)
def test_norm(kw):
    print(f"\n[case] {kw}", flush=True)
    kw = dict(kw)
    pad, shift, alias, no_y = kw.pop("pad", 0), kw.pop("shift", 0), kw.pop("alias", False), kw.pop("no_y", False)
    rows, d, g = kw["rows"], kw["width"], kw.get("group", kw["width"])
    dtype = kw.setdefault("dtype", "bf16")
    rdtype = kw.get("res_dtype", dtype)
    post, pre, gate = kw.setdefault("post", "rms"), kw.setdefault("pre", "none"), kw.setdefault("gate", "none")
    run, eps, scale = kw.setdefault("gate_run", 1), 1e-5, kw.get("scale", 1.0)
    rng = np.random.default_rng(d + rows)

    def home(n, t, mean=0.0):
        x = torch.zeros((n + 1) * (d + pad) + shift + 8, dtype=TD[t], device="cuda")[shift:].as_strided((n, d), (d + pad, 1))
        return x.copy_(torch.from_numpy(rng.standard_normal((n, d)) + mean).to(TD[t]))

    u = home(rows, dtype, 3.0)
    vec = lambda n: torch.from_numpy(1 + 0.3 * rng.standard_normal(n)).float().cuda()  # noqa: E731
    pw, pb = vec(g), vec(g) if post == "layer" else None
    hw, hb = vec(d), vec(d) if pre == "layer" else None
    z = home(-(-rows // run), dtype) if gate != "none" else None
    res = home(rows, rdtype) if kw.get("residual") else None
    sv = vec(d) if kw.get("scale_vec") else None
    y = None if no_y else home(rows, rdtype)
    h = home(rows, dtype) if pre != "none" else None
    strides = {f"{n}_row": d + pad for n in ("u", "gate", "res", "y", "h")}
    op = M.GateNorm(**kw, post_bias=pb is not None, pre_bias=hb is not None, eps=eps, **strides)
    res0 = None if res is None else _host(res)
    if alias:
        y = res
    op.run(u, pw if post != "none" else None, pb, z, res, sv, hw if pre != "none" else None, hb, y, h)
    if rows == 0:
        return

    x = _host(u)
    size = np.abs(x)
    on = np.ones_like(x)
    if z is not None:
        zz = _host(z)[np.arange(rows) // run]
        on = {"linear": zz, "silu": ref.silu(zz), "sigmoid": ref.sigmoid(zz)}[gate]
    if kw.get("gate_first"):
        x = x * on
    x, size = ref.norm(x.reshape(-1, g), post, _host(pw), None if pb is None else _host(pb), eps)
    x, size = x.reshape(rows, d), size.reshape(rows, d)
    if not kw.get("gate_first"):
        x, size = x * on, size * np.abs(on)
    f = scale * (1.0 if sv is None else _host(sv))
    x, size = x * f, size * np.abs(f)
    if res is not None:
        x, size = x + res0, size + np.abs(res0)
    t1 = (2 * 96 + 32) * U
    if y is not None:
        _near(_host(y), x, size, t1 + (R if rdtype == "bf16" else 0), "y")
    if h is not None:
        want, size2 = ref.norm(x, pre, _host(hw), None if hb is None else _host(hb), eps)
        # what x is off by, through the norm: its own place, the mean and the root
        r = 1 / np.sqrt(((x - (x.mean(-1, keepdims=True) if pre == "layer" else 0)) ** 2).mean(-1, keepdims=True) + eps)
        passed = t1 * (size + size.mean(-1, keepdims=True)) * r * np.abs(_host(hw))
        passed = passed + t1 * np.sqrt((size ** 2).mean(-1, keepdims=True)) * r * size2
        bound = (passed + t1 * size2) * (1 + R) + (R * np.abs(want) if dtype == "bf16" else 0)
        _near(_host(h), want, bound, 1.0, "h")


NORM_MANY = [
    # enough groups for two accesses per thread; ends inside an access; both types, also in place
    *[_case(rows=r, width=g * n, group=g, gate="silu") for g, r, n in ((9, 300, 7), (131, 150, 16), (250, 150, 16), (600, 260, 8),
                                                                      (1003, 260, 8), (2065, 257, 8), (4103, 257, 8))],
    *[_case(rows=r, width=g * n, group=g, gate="silu", dtype="f32", post="layer")
      for g, r, n in ((5, 300, 7), (67, 40, 16), (127, 40, 16), (258, 40, 8), (511, 40, 8), (1025, 40, 8), (2051, 40, 8))],
    *[_case(rows=300, width=d, dtype=t, residual=True, pre="layer", post="layer", gate="sigmoid", gate_run=7, alias=a, pad=1)
      for d in (13, 130, 515, 1537) for t, a in (("bf16", True), ("f32", False))],
]


@pytest.mark.parametrize("kw", NORM_MANY)
def test_norm_of_many_groups(kw):
    test_norm(kw)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("width", [3, 9, 129, 1027])
def test_rows_between_nan(dtype, width):
    """What lies beside the rows of a convolution and of a norm is no operand and stays as it is."""
    n, td = 70, TD[dtype]

    def home(value):
        return torch.full(((n + 2) * (width + 3),), value, dtype=td, device="cuda")

    def rows(flat):
        return flat[1:].as_strided((n, width), (width + 3, 1))

    x, y, h = home(float("nan")), home(5.0), home(5.0)
    dense = torch.randn(n, width, device="cuda").to(td)
    rows(x).copy_(dense)
    strides = {f"{k}_row": width + 3 for k in ("u", "res", "y", "h")}
    w = torch.rand(width, device="cuda")
    want, want_h = torch.empty_like(dense), torch.empty_like(dense)
    kw = dict(rows=n, width=width, dtype=dtype, residual=True, pre="rms")
    M.GateNorm(**kw, **strides).run(rows(x), w, residual=rows(x), pre_w=w, y=rows(y), h=rows(h))
    M.GateNorm(**kw).run(dense, w, residual=dense, pre_w=w, y=want, h=want_h)
    assert torch.equal(rows(y), want) and torch.equal(rows(h), want_h) and bool(torch.isfinite(want).all())
    taps = torch.randn(width, 4, device="cuda").to(td)
    win, left = torch.randn(1, 3, width, device="cuda").to(td), torch.full((2, 3, width), 5.0, device="cuda").to(td)
    kw = dict(tokens=n, seqs=1, channels=width, width=4, dtype=dtype, bias=False)
    out = home(5.0)
    M.TokenConv(**kw, x_row=width + 3, y_row=width + 3).run(rows(x), taps, None, win, left[:1], rows(out))
    M.TokenConv(**kw).run(dense, taps, None, win, win, want)  # in place
    assert torch.equal(rows(out), want) and torch.equal(left[:1], win) and bool((left[1] == 5.0).all())
    for flat in (y, h, out):
        rows(flat).fill_(5.0)
        assert bool((flat == 5.0).all())


def test_norm_rows_stay_apart():
    """A row of infinities or NaN, or of the type's largest values, changes no other row; a row of zeros norms to the bias."""
    for g in (64, 512):
        u = torch.randn(20, 512, device="cuda").bfloat16()
        w = torch.rand(g, device="cuda")
        op = M.GateNorm(rows=20, width=512, group=g)
        a, b = torch.empty_like(u), torch.empty_like(u)
        op.run(u, w, y=a)
        u[3], u[7], u[11] = float("nan"), float("inf"), 0.0
        op.run(u, w, y=b)
        keep = [i for i in range(20) if i not in (3, 7, 11)]
        assert torch.equal(a[keep], b[keep]) and bool((b[11] == 0).all())
        assert bool(torch.isnan(b[3]).all())


def test_descriptors_on_another_stream_and_device_errors():
    u = torch.randn(64, 256, device="cuda").bfloat16()
    w, y, y2 = torch.rand(256, device="cuda"), torch.empty_like(u), torch.empty_like(u)
    op = M.GateNorm(rows=64, width=256)
    op.run(u, w, y=y)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    op.run(u, w, y=y2, stream=s)
    torch.cuda.synchronize()
    assert torch.equal(y, y2)
    with pytest.raises(B.Conv2dError):
        op.run(u, w.cpu(), y=y)
