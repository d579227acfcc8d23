"""Softmax attention, rotary positions and cache pages against their float64 definitions (needs the GPU).

Tolerances are those of `oracle.seqmix.softmax_bound`, point by point; those of rotary positions are derived at `_near_rotary`;
pages are whole numbers and equal.
"""
import numpy as np
import pytest
import torch

from oracle import seqmix as ref
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


def _near(got, want, bound, what):
    fine = np.isfinite(want)
    assert np.array_equal(np.isfinite(got), fine), f"{what}: finite in other places"
    if fine.any():
        worst = float((np.abs(got - want)[fine] / bound[fine]).max())
        print(f"  {what}: {worst:.3f} of the bound", flush=True)
        assert worst <= 1.0, f"{what}: {worst:.3g} times the bound"


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Soft:
    """One problem: `new` rows and `keys` keys per sequence, its tensors strided or shifted as asked, and its definition."""

    def __init__(self, new, keys=None, heads=2, kv_heads=1, dk=64, dv=64, dtype="bf16", mask="causal", page=0, seed=0, shift=0,
                 pad=0, heads_outer=False, uniform=None, scale=None, spare=3, tree=None, skip=(), page_stride=None, qscale=1.0):
        rng = np.random.default_rng(seed)
        keys = list(new) if keys is None else keys
        self.new, self.keys, self.heads, self.mask, self.dtype, self.dk, self.page = new, keys, heads, mask, dtype, dk, page
        n, m, td = sum(new), len(new), TD[dtype]
        self.n, self.skip, self.scale = n, skip, dk ** -0.5 if scale is None else scale

        def dev(rows, h, d):  # a strided home for [rows, h, d]
            if heads_outer:
                flat = torch.zeros(h * (rows + 1) * (d + pad) + shift + 16, dtype=td, device="cuda")
                return flat[shift:].as_strided((rows, h, d), (d + pad, (rows + 1) * (d + pad), 1))
            flat = torch.zeros((rows + 1) * (h * d + pad) + shift + 16, dtype=td, device="cuda")
            return flat[shift:].as_strided((rows, h, d), (h * d + pad, d, 1))

        def fill(t, s=1.0):
            return t.copy_(torch.from_numpy(rng.standard_normal(tuple(t.shape)) * s).to(td))

        self.q, self.o = fill(dev(n, heads, dk), qscale), dev(n, heads, dv)
        self.o.fill_(7.0)
        uniform = len(set(new)) == 1 if uniform is None else uniform
        self.off = None if uniform else torch.tensor([0] + list(new), device="cuda").cumsum(0)
        self.tree_host = self.tree = None
        if mask == "tree":
            self.tree_host = [int(rng.integers(0, 2 ** 63)) * 2 + int(rng.integers(0, 2)) for _ in range(n)] if tree is None else tree
            self.tree = torch.tensor([t - (1 << 64) if t >= 1 << 63 else t for t in self.tree_host], device="cuda")
        self.koff = self.lens = self.table = self.slot = None
        slots, more = m, {}
        if page:
            slots = m + spare
            need = [-(-t // page) for t in keys]
            pages, most = sum(need) + 2, max(need + [1]) + 1
            order = rng.permutation(pages)
            places = rng.permutation(slots)[:m]
            table = np.full((slots, most), -1)
            at = 0
            for s, c in zip(places, need):
                table[s, :c] = order[at:at + c]
                at += c
            lens = np.zeros(slots, int)
            lens[places] = keys
            self.where = [(s, table[s, :c]) for s, c in zip(places, need)]
            places = [slots + 5 if i in skip else s for i, s in enumerate(places)]
            self.lens, self.table, self.slot = _ints(lens.tolist()), _ints(table.tolist()), _ints([int(s) for s in places])

            def cache(d):
                if page_stride:  # pages far apart
                    flat = torch.empty((pages - 1) * page_stride + page * kv_heads * d, dtype=td, device="cuda")
                    return flat.as_strided((pages, page, kv_heads, d), (page_stride, kv_heads * d, d, 1))
                if heads_outer:  # [pages][heads][page][d]
                    flat = torch.zeros(pages * kv_heads * page * d + shift + 16, dtype=td, device="cuda")
                    return flat[shift:].as_strided((pages, page, kv_heads, d), (kv_heads * page * d, d, page * d, 1))
                flat = torch.zeros(pages * page * kv_heads * d + shift + 16, dtype=td, device="cuda")
                return flat[shift:shift + pages * page * kv_heads * d].view(pages, page, kv_heads, d)

            self.k, self.v = fill(cache(dk)), fill(cache(dv))
            more = dict(page=page, pages=pages, max_pages=most)
        else:
            self.k, self.v = fill(dev(sum(keys), kv_heads, dk)), fill(dev(sum(keys), kv_heads, dv))
            if keys != list(new):
                self.koff = torch.tensor([0] + list(keys), device="cuda").cumsum(0)
                more = dict(key_tokens=sum(keys))
            if skip:
                self.slot = _ints([-1 if i in skip else i for i in range(m)])
        self.op = M.SoftmaxAttention(
            tokens=n, seqs=m, slots=slots, heads=heads, kv_heads=kv_heads, dk=dk, dv=dv, dtype=dtype, mask=mask,
            scale=self.scale, q_strides=self.q.stride()[:2], o_strides=self.o.stride()[:2],
            k_strides=self.k.stride()[:-1], v_strides=self.v.stride()[:-1], **more)

    def run(self, **kw):
        self.op.run(self.q, self.k, self.v, self.o, offsets=self.off, key_offsets=self.koff, slot_index=self.slot, lens=self.lens,
                    table=self.table, tree=self.tree, **kw)
        return self

    def parts(self):
        """bf16 parts of a weight."""
        return 2 if self.op.plan().kernel == M.SEQMIX_KERNEL_STEP else 1

    def held(self, i):
        """Keys and values of sequence i."""
        if self.page:
            at = torch.tensor(self.where[i][1], device="cuda", dtype=torch.long)
            return (_host(t[at].flatten(0, 1)[:self.keys[i]]) for t in (self.k, self.v))
        first = sum(self.keys[:i])
        return (_host(t[first:first + self.keys[i]]) for t in (self.k, self.v))

    def check(self):
        got, q, first = _host(self.o), _host(self.q), 0
        for i, n in enumerate(self.new):
            rows = slice(first, first + n)
            first += n
            if i in self.skip:
                assert (got[rows] == 7.0).all(), "rows of a skipped sequence were written"
                continue
            if not n:
                continue
            k, v = self.held(i)
            on = ref.sees(self.mask, n, self.keys[i], None if self.tree_host is None else self.tree_host[rows])
            o, o_abs, most = ref.softmax_attention(q[rows], k, v, on, self.scale)
            bound = ref.softmax_bound(o, o_abs, most, self.keys[i], self.dk, self.dtype, self.parts())
            _near(got[rows], o, bound, f"sequence {i}")
            assert (got[rows][~on.any(1)] == 0).all(), "rows that see nothing"
        return self


def _case(**kw):
    return pytest.param(kw, id="-".join(f"{k}{v}" for k, v in kw.items()).replace(" ", ""))


CASES = [
    # around the edges of tiles, both types
    *[_case(new=[t], dtype=d) for t in (1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200) for d in ("bf16", "f32")],
    # head sizes: those of the kernels, between them, odd, one
    *[_case(new=[70], dk=dk, dv=dv, dtype=d) for d in ("bf16", "f32") for dk, dv in (
        (128, 128), (64, 128), (128, 64), (256, 256), (64, 256), (256, 64), (128, 256), (256, 128), (192, 128), (80, 112),
        (96, 96), (33, 71), (100, 30), (1, 1), (200, 132), (129, 255), (8, 8))],
    # shared heads; rows of few tokens are packed
    *[_case(new=[5, 7, 1, 0, 4], heads=12, kv_heads=k, dk=128, dv=128) for k in (1, 2, 3, 4, 6, 12)],
    _case(new=[2] * 6, heads=10, kv_heads=2, dk=48, dv=40, dtype="f32"),
    _case(new=[3] * 3, heads=64, kv_heads=1, dk=64, dv=64),
    # ragged, empty sequences at every place
    _case(new=[0, 70, 1, 0, 0, 200, 64, 3, 0], heads=3, kv_heads=3, dk=64, dv=96),
    _case(new=[0, 70, 1, 0, 0, 200, 64, 3, 0], heads=4, kv_heads=2, dk=40, dv=128, dtype="f32"),
    _case(new=[90] * 3, uniform=False),
    # other numbers of keys than rows: more, fewer, none
    _case(new=[40, 3, 20, 64], keys=[40, 100, 0, 10]),
    _case(new=[40, 3, 20, 64], keys=[300, 2, 21, 64], dtype="f32"),
    _case(new=[40, 3, 20, 64], keys=[300, 2, 0, 64], mask="full"),
    _case(new=[100, 2], keys=[90, 500], mask="full", dtype="f32", dk=80, dv=24),
    _case(new=[4, 0], keys=[0, 0], mask="full"),
    # pages that end inside tiles, and that hold many
    *[_case(new=[40, 3, 0, 65], keys=[300, 77, 20, 65], page=p) for p in (1, 2, 16, 64, 128, 512)],
    _case(new=[40, 3, 0, 65], keys=[300, 77, 20, 65], page=16, dtype="f32", heads=4, kv_heads=2, dk=128, dv=128),
    _case(new=[40, 3, 0, 65], keys=[300, 77, 20, 65], page=32, dk=72, dv=100, mask="full"),
    _case(new=[40, 3, 0, 65], keys=[300, 77, 20, 65], page=32, heads=4, kv_heads=2, heads_outer=True),
    # single tokens over a cache
    *[_case(new=[1] * 5, keys=[1, 700, 64, 65, 333], heads=h, kv_heads=k, dk=128, dv=128, page=16, dtype=d)
      for h, k in ((4, 4), (8, 2), (16, 1), (6, 2)) for d in ("bf16", "f32")],
    _case(new=[1] * 2, keys=[5000, 3000], heads=4, kv_heads=1, dk=128, dv=128, page=64),
    _case(new=[1], keys=[9001], heads=1, kv_heads=1, dk=64, dv=64, page=128, dtype="f32"),
    _case(new=[1, 1], keys=[3001, 40], heads=2, kv_heads=2, dk=256, dv=256, page=16),
    _case(new=[1, 1], keys=[301, 40], heads=2, kv_heads=2, dk=99, dv=37, page=16),
    _case(new=[1, 1], keys=[3001, 0], heads=3, kv_heads=1, dk=192, dv=128, page=32),
    # trees of drafted tokens; masks that leave rows empty (nothing went before)
    *[_case(new=[t] * 3, keys=[t, t + 50, t + 700], mask="tree", heads=8, kv_heads=2, dk=128, dv=128, page=16)
      for t in (2, 5, 24, 33, 63, 64)],
    _case(new=[7, 64, 1, 0, 30], keys=[7, 90, 1, 4, 500], mask="tree", heads=6, kv_heads=2, dk=80, dv=64, dtype="f32", page=8),
    _case(new=[6, 6], keys=[6, 106], mask="tree", tree=[0, 1, 0, 2, 32, 1 << 63, 0, 1, 3, 1 << 40, 63, 0]),
    _case(new=[70, 5], keys=[100, 3], mask="tree"),  # more rows than a mask has bits; fewer keys than rows
    # scales: negative, none, large scores
    _case(new=[50], scale=-0.3), _case(new=[50], scale=0.0), _case(new=[50], scale=0.0, dtype="f32"),
    _case(new=[90], qscale=20.0, dk=128), _case(new=[90], qscale=20.0, dtype="f32"), _case(new=[90], scale=1e-30),
    # strides, alignments and orders
    *[_case(new=[70, 9], heads=4, kv_heads=2, shift=s, pad=p, heads_outer=o, dtype=d) for d in ("bf16", "f32")
      for s, p, o in ((0, 8, False), (1, 3, False), (3, 5, True), (0, 0, True))],
    _case(new=[5, 9], keys=[33, 200], heads=4, kv_heads=2, shift=1, page=16),
    # skipped sequences
    _case(new=[20, 30, 5], skip=(1,)), _case(new=[20, 30, 5], keys=[50, 30, 5], skip=(0, 2), page=16),
]


@pytest.mark.parametrize("kw", CASES)
def test_softmax(kw):
    Soft(**kw).run().check()


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("mask", ("causal", "tree"))
@pytest.mark.parametrize("page", (0, 16))
def test_what_is_not_seen_does_not_matter(dtype, mask, page):
    """Keys and values that are infinite or NaN reach the rows that see them, and no others."""
    n, keys = 40, 200
    tree = [(1 << (j + 1)) - 1 & ~(1 << 20) for j in range(n)]  # all up to itself, but never number 20
    p = Soft([n, n], keys=[keys, n], heads=4, kv_heads=2, dk=64, dv=80, dtype=dtype, mask=mask, page=page, tree=tree * 2)
    bad = [float("nan"), float("inf"), float("-inf")]

    def at(t, i, j):  # row of key j of sequence i
        if page:
            return t[int(p.where[i][1][j // page]), j % page]
        return t[sum(p.keys[:i]) + j]

    for x, value in enumerate(bad):
        at(p.v, 0, keys - n + 20)[0, x] = value  # the row of token 20
        at(p.v, 1, 20)[1, x] = value
        at(p.k, 0, keys - 1)[0, x] = value       # the last token's
    if page:  # behind the ends
        at(p.k, 1, 39)  # (exists)
        last = int(p.where[1][1][-1])
        p.k[last, n % page:] = float("nan")
        p.v[last, n % page:] = float("inf")
    p.run()
    got, q, first = _host(p.o), _host(p.q), 0
    for i in range(2):
        k, v = p.held(i)
        on = ref.sees(mask, n, p.keys[i], tree)
        o, o_abs, most = ref.softmax_attention(q[first:first + n], k, v, on, p.scale)
        rows = got[first:first + n]
        first += n
        fine = np.isfinite(o)
        assert np.array_equal(np.isfinite(rows), fine)
        assert np.isnan(rows[~fine]).all()
        bound = ref.softmax_bound(o, o_abs, most, p.keys[i], p.dk, dtype, p.parts())
        assert (np.abs(rows - o)[fine] <= bound[fine]).all()


# Few tiles over many keys: bf16 rows over more than 1024 keys (single tokens 1536), fp32 rows over more than 64, are divided and joined.
DIVIDED = [
    _case(new=[300, 7], keys=[2000, 900], heads=4, kv_heads=2, dk=128, dv=128, page=16),
    _case(new=[130], keys=[5000], mask="full", heads=2, kv_heads=1, dk=64, dv=256),
    _case(new=[40, 3, 0], keys=[2500, 64, 30], mask="full", heads=8, kv_heads=1, dk=128, dv=128),
    _case(new=[130, 40], keys=[4500, 40], heads=3, kv_heads=3, dk=99, dv=37, page=16),
    _case(new=[1500], heads=1, kv_heads=1, dk=80, dv=112),
    _case(new=[1500, 2], heads=2, kv_heads=1, dk=64, dv=64, dtype="f32"),
    _case(new=[200, 1], keys=[1300, 700], heads=3, kv_heads=1, dk=33, dv=70, dtype="f32", page=8),
    *[_case(new=[24] * 3, keys=[3000, 24, 1900], mask="tree", heads=8, kv_heads=2, dk=d, dv=d, page=32) for d in (64, 128, 192)],
    *[_case(new=[t] * 2, keys=[6000, 1600], heads=8, kv_heads=2, dk=128, dv=128, page=16, dtype=d) for t in (1, 3, 8) for d in ("bf16", "f32")],
    _case(new=[1] * 2, keys=[40000, 1], heads=4, kv_heads=4, dk=64, dv=64, page=64),   # 512 shares' worth of parts for one row
    _case(new=[1] * 2, keys=[4000, 2000], heads=5, kv_heads=1, dk=127, dv=63, page=16),
    _case(new=[1] * 70, keys=[3000 if i % 9 == 0 else i for i in range(70)], heads=2, kv_heads=2, dk=64, dv=64, page=16),
    _case(new=[2] * 70, keys=[1700 if i == 66 else 2 for i in range(70)], heads=2, kv_heads=1, dk=64, dv=64, page=16, skip=(65, 67)),
    _case(new=[66] * 3 + [0, 140], keys=[66, 1500, 4000, 9, 200], heads=4, kv_heads=1, dk=128, dv=64, page=64, skip=(1,)),
]


# Rows that are no multiple of 16 bytes, of each pair of kernels' sizes: in one page a tile or several, packed, a few or many rows.
ODD = [_case(new=new, keys=keys, heads=4, kv_heads=2, dk=dk, dv=dv, dtype=d, page=page, shift=shift)
       for (dk, dv), (new, keys, page, shift) in zip(
           ((33, 57), (33, 100), (35, 131), (99, 61), (127, 127), (101, 255), (131, 64), (203, 99), (231, 233), (9, 5), (64, 66), (82, 112)) * 3,
           (([70, 9], [170, 300], 16, 0), ([1, 1, 1], [500, 1, 67], 64, 1), ([130], None, 0, 0), ([3, 1], [90, 700], 8, 0),
            ([40, 90], [333, 90], 128, 1)) * 8)
       for d in ("bf16", "f32")]


# Dims around three quarters of the kernels' sizes, few rows, keys that end inside 8.
ODD += [_case(new=[1, 3], keys=[301, 41], heads=4, kv_heads=2, dk=dk, dv=dv, dtype="f32", page=16, shift=0)
        for dk, dv in ((48, 48), (80, 80), (96, 96), (97, 97), (96, 128), (128, 96), (192, 192), (193, 192), (192, 193), (256, 100))]


@pytest.mark.parametrize("kw", ODD)
def test_odd_rows(kw):
    p = Soft(**kw)
    if p.page:  # what lies behind the ends is never read
        for i, (_, pages) in enumerate(p.where):
            if p.keys[i] % p.page:
                for t in (p.k, p.v):
                    t[int(pages[-1]), p.keys[i] % p.page:] = float("nan")
    p.run().check()


@pytest.mark.parametrize("kw", DIVIDED)
def test_divided(kw):
    p = Soft(**kw)
    assert p.op.plan().shares > 0
    p.run().check()


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("n,heads", ((3, 4), (40, 2), (150, 2)))
def test_divided_rows_and_values_that_are_not_finite(dtype, n, heads):
    """One value early and one late of many keys: the rows that see them are NaN there, whichever part holds them, and no others."""
    keys = 5000
    p = Soft([n], keys=[keys], heads=heads, kv_heads=heads // 2, dk=64, dv=64, dtype=dtype, page=16)
    where = p.where[0][1]

    def at(t, j):
        return t[int(where[j // 16]), j % 16]

    at(p.v, 100)[0, 5] = float("inf")            # seen by all rows
    at(p.v, keys - 1)[heads // 2 - 1, 9] = float("nan")  # by the last row only
    at(p.v, keys - 2)[0, 11] = float("-inf")     # by the last two
    assert p.op.plan().shares > 0
    p.run()
    got, q = _host(p.o), _host(p.q)
    k, v = p.held(0)
    on = ref.sees("causal", n, keys)
    o, o_abs, most = ref.softmax_attention(q, k, v, on, p.scale)
    fine = np.isfinite(o)
    assert not fine.all() and np.array_equal(np.isfinite(got), fine) and np.isnan(got[~fine]).all()
    bound = ref.softmax_bound(o, o_abs, most, keys, p.dk, dtype, p.parts())
    assert (np.abs(got - o)[fine] <= bound[fine]).all()


def test_query_that_is_not_finite_stays_with_its_row():
    p = Soft([50, 30], heads=2, kv_heads=1)
    p.q[7, 1, 3] = float("nan")
    p.q[60, 0, 0] = float("inf")
    p.run()
    bad = torch.isnan(p.o).all(-1)
    assert bad.nonzero().tolist() == [[7, 1], [60, 0]]
    assert torch.isfinite(p.o[~bad]).all()


def test_far_pages():
    """A cache whose offsets pass 32 bits."""
    p = Soft([2, 1], keys=[600, 400], heads=4, kv_heads=2, dk=64, dv=64, page=16, page_stride=1 << 26)
    assert p.k.stride(0) * (p.k.shape[0] - 1) > 1 << 31
    p.run().check()


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("stride", ((1 << 18) + 8, (1 << 22) + 1))
def test_far_rows(stride, dtype):
    """Packed keys and values whose rows lie further apart than 32-bit offsets of a tile reach."""
    p = Soft([5, 40], keys=[20, 70], heads=2, kv_heads=1, dk=64, dv=64, dtype=dtype)
    for name in ("k", "v"):
        old = getattr(p, name)
        flat = torch.empty(89 * stride + 64, dtype=old.dtype, device="cuda")
        new = flat.as_strided((90, 1, 64), (stride, 64, 1))
        setattr(p, name, new.copy_(old))
    p.op = M.SoftmaxAttention(tokens=45, seqs=2, heads=2, kv_heads=1, dk=64, dv=64, dtype=dtype, scale=p.scale, key_tokens=90,
                              q_strides=p.q.stride()[:2], o_strides=p.o.stride()[:2], k_strides=(stride, 64), v_strides=(stride, 64))
    p.run().check()


@pytest.mark.parametrize("kw", [dict(new=[1] * 1100, page=16, heads=2, kv_heads=1), dict(new=[40] + [2] * 1030 + [0, 90], heads=1, kv_heads=1),
                                dict(new=[3] * 1050, page=8, heads=2, kv_heads=2, mask="tree", dtype="f32")])
def test_many_sequences(kw):
    """More sequences than a wave looks over for shares."""
    more = kw.get("page") and dict(keys=[n + (i * 37) % 90 for i, n in enumerate(kw["new"])])
    p = Soft(dk=64, dv=64, **kw, **(more or {}))
    assert p.op.plan().shares == 0
    p.run().check()


def test_two_graphs_of_one_descriptor():
    """Graphs that share a workspace, replayed one after the other with an eager call between them."""
    p = Soft([1] * 2, keys=[9000, 3000], heads=8, kv_heads=2, dk=128, dv=128, page=16)
    p.op.reserve()
    p.run()
    outs, graphs = [torch.empty_like(p.o) for _ in range(2)], []
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for o in outs:
        p.o = o
        g = torch.cuda.CUDAGraph()
        with torch.cuda.stream(side), torch.cuda.graph(g, stream=side):
            p.run()
        graphs.append(g)
    p.o = torch.empty_like(outs[0])
    for seed in range(3):
        p.q.copy_(torch.randn(p.q.shape, device="cuda", generator=torch.Generator("cuda").manual_seed(seed)))
        for o in outs:
            o.zero_()
        graphs[0].replay()
        p.run()
        graphs[1].replay()
        graphs[0].replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0], p.o) and torch.equal(outs[1], p.o)
    p.check()


@pytest.mark.parametrize("kw", [dict(new=[7, 300, 0, 20]), dict(new=[1, 1, 1], keys=[700, 20, 3000], page=16),
                                dict(new=[9, 9], keys=[2000, 9], mask="tree", page=16)])
def test_bad_lengths_and_pages_stay_inside(kw):
    """Offsets, lengths and page numbers out of range give some result; neighbours in memory are not written."""
    p = Soft(heads=4, kv_heads=2, dk=64, dv=64, **kw)
    p.run()
    room = torch.full((p.o.numel() + 4096,), 5.0, dtype=p.o.dtype, device="cuda")
    p.o = room[2048:2048 + p.o.numel()].view(p.o.shape)
    if p.page:
        p.table.copy_(torch.randint(-2 ** 31, 2 ** 31 - 1, p.table.shape, device="cuda"))
        p.lens.copy_(torch.randint(-5, 2 ** 31 - 1, p.lens.shape, device="cuda"))
        p.slot[0] = 2 ** 31 - 1
        p.run()
        assert (room[:2048] == 5).all() and (room[-2048:] == 5).all()
    for off in ([0, 10 ** 12, -7, 5, 4], [5, 4, 3, 2, 1], [-2 ** 62, 2 ** 62, -2 ** 62, 2 ** 62, 0]):
        p.off = torch.tensor(off[:len(p.new)] + off[-1:], device="cuda")
        p.run()
        torch.cuda.synchronize()
        assert (room[:2048] == 5).all() and (room[-2048:] == 5).all()


def test_rows_behind_the_last_sequence_are_left():
    p = Soft([40, 24, 16], heads=2, kv_heads=1)
    p.off = torch.tensor([0, 40, 64, 64], device="cuda")
    p.run()
    assert (p.o[64:] == 7).all() and (p.o[:64] != 7).any(-1).all()


def test_results_repeat():
    for kw in (dict(new=[1] * 3, keys=[5000, 70, 900], page=16), dict(new=[300, 7], keys=[2000, 900], page=16)):
        p = Soft(heads=8, kv_heads=2, dk=128, dv=128, **kw).run()
        first = p.o.clone()
        for _ in range(4):
            assert torch.equal(p.run().o, first)


@pytest.mark.parametrize("kw", [dict(new=[1] * 2, keys=[9000, 500], page=16), dict(new=[200, 70], keys=[3000, 70], page=16),
                                dict(new=[300])])
def test_captured(kw):
    """Replays with new inputs, between eager calls of the same descriptor and of others."""
    p = Soft(heads=8, kv_heads=2, dk=128, dv=128, **kw)
    p.op.reserve()
    p.run()
    g = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side), torch.cuda.graph(g, stream=side):
        p.run()
    for seed in range(4):
        torch.manual_seed(seed)
        p.q.copy_(torch.randn(p.q.shape, device="cuda"))
        p.run()
        want = p.o.clone()
        p.o.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(p.o, want)
        p.q.add_(1)
        p.run()


def test_another_stream():
    p = Soft([1] * 4, keys=[4000, 30, 600, 7000], heads=8, kv_heads=2, dk=128, dv=128, page=16).run()
    want = p.o.clone()
    s = torch.cuda.Stream()
    for _ in range(5):
        p.o.zero_()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            p.run()
        torch.cuda.current_stream().wait_stream(s)
        assert torch.equal(p.o, want)
        assert torch.equal(p.run(stream=torch.cuda.current_stream()).o, want)


# ------------------------------------------------------------------ rotary positions
def _near_rotary(got, x, want, layout, rot, dtype, amplitude, what):
    """The fraction of a turn is rounded to fp32, and doubled exactly: 2^-24 turns, 2 pi u radians; sine and cosine are off by as
    much and 2 ulp (2 u), their product with the amplitude, each product and the sum by u: (2 pi + 6) u (|a| + |b|)
    |amplitude|.  bf16 rounds once."""
    size = np.abs(x).copy()
    if layout == "half":
        both = size[..., :rot // 2] + size[..., rot // 2:rot]
        size[..., :rot // 2], size[..., rot // 2:rot] = both, both
    else:
        both = size[..., 0:rot:2] + size[..., 1:rot:2]
        size[..., 0:rot:2], size[..., 1:rot:2] = both, both
    _near(got, want, (2 * np.pi + 6) * U * size * max(1.0, abs(amplitude)) * (1 + R) + (R * np.abs(want) if dtype == "bf16" else 0)
          + 1e-37, what)


ROTARY = [
    _case(), _case(dtype="f32"), _case(layout="interleaved"), _case(layout="interleaved", dtype="f32"),
    _case(tokens=1), _case(tokens=1030, heads=2), _case(tokens=1027, heads=3, kv_heads=1, dtype="f32", page=16),
    _case(page=16), _case(page=1, tokens=70), _case(page=64, dtype="f32", amplitude=1.3, dv=112), _case(page=32, both=True),
    *[_case(dk=dk, rot=rot, layout=lay, dtype=d, page=16, dv=33) for lay in ("half", "interleaved") for d in ("bf16", "f32")
      for dk, rot in ((64, 32), (80, 50), (33, 6), (100, 100), (2, 2), (1, 0), (256, 254), (70, 0), (18, 18))],
    _case(heads=5, kv_heads=0), _case(heads=0, kv_heads=3), _case(shift=1, pad=3), _case(shift=3, pad=1, page=16, dtype="f32"),
    _case(in_place=True), _case(in_place=True, layout="interleaved", dk=50, rot=22), _case(far=2 ** 31 - 1), _case(far=2 ** 31 - 1, dtype="f32"),
    _case(negative=True, dtype="f32"), _case(heads_outer=True, page=16, kv_heads=3),
]


@pytest.mark.parametrize("kw", ROTARY)
def test_rotary(kw):
    kw = dict(dict(tokens=37, heads=4, kv_heads=2, dk=64, dv=64, layout="half", dtype="bf16", page=0, amplitude=1.0, shift=0,
                   pad=0, in_place=False, both=False, far=40000, negative=False, heads_outer=False), **kw)
    n, h, hk, dk, dv, dtype, page, layout = (kw[x] for x in ("tokens", "heads", "kv_heads", "dk", "dv", "dtype", "page", "layout"))
    rot, amp, td, rng = kw.get("rot", dk), kw["amplitude"], TD[dtype], np.random.default_rng(1)

    def dev(heads, d, fill=True):
        row = heads * d + kw["pad"]
        flat = torch.zeros(n * row + kw["shift"] + 16, dtype=td, device="cuda")
        t = flat[kw["shift"]:].as_strided((n, heads, d), (row, d, 1))
        return t.copy_(torch.from_numpy(rng.standard_normal((n, heads, d))).to(td)) if fill else t

    q, k, v = dev(h, dk), dev(hk, dk), dev(hk, dv)
    q0, k0 = _host(q), _host(k)
    qo, ko = (q, k) if kw["in_place"] else (dev(h, dk, False), dev(hk, dk, False))
    position = torch.from_numpy(rng.integers(0, kw["far"], n, endpoint=True).astype(np.int32)).cuda()
    position[-1] = kw["far"]
    if kw["negative"]:
        position.neg_()
    freqs = M.rotary_frequencies(rot, factor=4.0, trained=2048)
    pages = n // page + 2 if page else 0
    place = kc = vc = kc0 = vc0 = None
    if page:
        place = torch.from_numpy(rng.permutation(pages * page)[:n].astype(np.int32)).cuda()
        if n > 3:
            place[1], place[3] = -1, pages * page  # not stored
        kc, vc = (torch.randn(pages, page, hk, d, device="cuda").to(td) for d in (dk, dv))
        if kw["heads_outer"]:
            kc, vc = (t.transpose(1, 2).contiguous().transpose(1, 2) for t in (kc, vc))
        kc0, vc0 = _host(kc), _host(vc)
    op = M.Rotary(tokens=n, heads=h, kv_heads=hk, dk=dk, dv=dv, rot=rot, layout=layout, dtype=dtype, amplitude=amp, page=page,
                  pages=pages, q_strides=q.stride()[:2], k_strides=k.stride()[:2], v_strides=v.stride()[:2],
                  q_out_strides=qo.stride()[:2], k_out_strides=ko.stride()[:2],
                  k_cache_strides=kc.stride()[:3] if page else None, v_cache_strides=vc.stride()[:3] if page else None)
    with_out = not page or kw["both"]
    op.run(q if h else None, k if hk else None, v if page else None, position, freqs, qo if h else None, ko if hk and with_out else None,
           kc, vc, place)
    pos, f = position.cpu().numpy(), freqs.cpu().numpy()
    if h:
        _near_rotary(_host(qo), q0, ref.rotary(q0, pos, f, rot, layout, amp), layout, rot, dtype, amp, "q")
    if hk:
        turned = ref.rotary(k0, pos, f, rot, layout, amp)
        if with_out:
            _near_rotary(_host(ko), k0, turned, layout, rot, dtype, amp, "k")
        if page:
            at = place.cpu().numpy()
            on = (at >= 0) & (at < pages * page)
            got = _host(kc)[at[on] // page, at[on] % page]
            _near_rotary(got, k0[on], turned[on], layout, rot, dtype, amp, "k in the cache")
            assert np.array_equal(_host(vc)[at[on] // page, at[on] % page], _host(v)[on])
            rest = np.ones((pages, page), bool)
            rest[at[on] // page, at[on] % page] = False
            assert np.array_equal(_host(kc)[rest], kc0[rest]) and np.array_equal(_host(vc)[rest], vc0[rest])


# ------------------------------------------------------------------ pages
class Pool:
    def __init__(self, slots, pages, max_pages, page, seed=0):
        self.rng = np.random.default_rng(seed)
        self.page, self.slots, self.pages, self.max_pages = page, slots, pages, max_pages
        self.t = M.CachePages.empty(slots, pages, max_pages)
        self.t[2].copy_(torch.from_numpy(self.rng.permutation(pages)))
        self.want = ref.Pages(*(x.tolist() for x in self.t[:3]), 0, page)

    def move(self, slots, new, kept=None, uniform=None, pad=0):
        """slots: None for a skipped one."""
        n, m = sum(new) + pad, len(slots)
        uniform = (len(set(new)) == 1 and not pad) if uniform is None else uniform
        op = M.CachePages(tokens=n, seqs=m, slots=self.slots, page=self.page, pages=self.pages, max_pages=self.max_pages)
        place, position = torch.full((n,), 99, dtype=torch.int32, device="cuda"), torch.full((n,), 99, dtype=torch.int32, device="cuda")
        admitted = torch.full((m,), 99, dtype=torch.int32, device="cuda")
        off = None if uniform else torch.tensor([0] + list(new), device="cuda").cumsum(0)
        index = _ints([self.slots + 1 if s is None else int(s) for s in slots])
        op.run(None if kept is None else _ints(kept), *self.t, place, position, admitted, offsets=off, slot_index=index)
        want = self.want.move(slots, kept, new)
        assert place.tolist() == want[0] + [-1] * pad
        assert position.tolist() == want[1] + [0] * pad
        assert admitted.tolist() == want[2]
        assert self.t[0].tolist() == self.want.lens
        assert self.t[1].tolist() == self.want.table
        assert self.t[2].tolist() == self.want.free
        assert self.t[3].tolist() == [self.want.taken]
        return admitted


def test_pages_of_a_serving_loop():
    """Requests come with prompts, go on by tokens and drafts, lose refused drafts, end; the pool runs out and empties."""
    p = Pool(slots=9, pages=40, max_pages=12, page=16)
    p.move([3, 0, 8], [100, 16, 1])
    p.move([0, 3, 8], [1, 1, 1])
    p.move([3, 8, 0], [8, 8, 8])
    p.move([3, 8, 0], [8, 8, 8], kept=[103, 2, 18])
    p.move([1, None, 5], [190, 5, 180])
    p.move([2, 4, 3], [0, 300, 1])           # longer than a row of the table
    p.move([2, 6, 8], [150, 160, 1])         # more than is left: those that need pages from there on
    p.move([3, 0], [0, 0], kept=[0, 5])      # one ends
    p.move([6, 2, 3], [10, 20, 0], kept=[5, 5, 5])
    p.move(list(range(9)), [0] * 9, kept=[0] * 9)
    assert p.t[3].item() == 0 and sorted(p.t[2].tolist()) == list(range(40))


@pytest.mark.parametrize("page", (1, 2, 64, 4096))
def test_pages_of_many_sizes(page):
    p = Pool(slots=50, pages=400, max_pages=20, page=page)
    rng = np.random.default_rng(page)
    for _ in range(6):
        slots = [int(s) if rng.random() < 0.9 else None for s in rng.permutation(50)[:int(rng.integers(1, 50))]]
        new = [int(x) for x in rng.integers(0, 3 * min(page, 300) + 2, len(slots))]
        p.move(slots, new, kept=[int(x) for x in rng.integers(-3, 9 * page, len(slots))] if rng.random() < 0.7 else None)


def test_pages_of_many_requests():
    """More requests than a workgroup has threads, and rows that a second launch places."""
    p = Pool(slots=2600, pages=3000, max_pages=3, page=16)
    order = [int(x) for x in np.random.default_rng(2).permutation(2600)]
    p.move(order[:2500], [1] * 2500)
    p.move(order[100:2550], [17] * 2450)                  # the pool runs out
    p.move(order[:1200], [2] * 1200, kept=[0] * 1200)
    p.move(order[:1000], [5, 0, 9, 30] * 250, kept=[3] * 1000)
    p.move(order[50:60], [900, 0, 0, 40, 4000, 1, 30, 7, 20, 48])


def test_rows_of_no_sequence_have_no_place():
    p = Pool(slots=4, pages=40, max_pages=12, page=16)
    p.move([0, 2], [20, 3], pad=9)
    p.move([2, 0], [30, 0], pad=5000)


def test_bad_pages_stay_inside():
    """Lengths, counts, slots and offsets that lie: the call ends, and nothing around its tensors changes."""
    slots, pages, most = 6, 30, 5
    room = [torch.full((s + 2048,), 77, dtype=torch.int32, device="cuda") for s in (slots, slots * most, pages, 1, 50, 50, 4)]
    lens, table, free, taken, place, position, admitted = (r[1024:-1024] for r in room)
    op = M.CachePages(tokens=50, seqs=4, slots=slots, page=16, pages=pages, max_pages=most)
    for seed in range(6):
        torch.manual_seed(seed)
        for t in (lens, table, free, taken):
            t.copy_(torch.randint(-2 ** 31, 2 ** 31 - 1, t.shape, device="cuda"))
        off = torch.tensor([[0, 9, 3, 60, 50], [0, 10 ** 12, -5, 50, 2], [50, 40, 30, 20, 10]][seed % 3], device="cuda")
        op.run(_ints([5, -9, 2 ** 31 - 1, 0]), lens, table.view(slots, most), free, taken, place, position, admitted, offsets=off,
               slot_index=_ints([1, 1, 2 ** 31 - 1, 5] if seed % 2 else [0, 3, 4, 5]))
        torch.cuda.synchronize()
        assert all((r[:1024] == 77).all() and (r[-1024:] == 77).all() for r in room)
        assert ((place >= -1) & (place < pages * 16)).all() and 0 <= taken.item() <= pages


# ------------------------------------------------------------------ together
def test_a_layer_served_with_them():
    """Prompts, tokens one by one, drafts and refused drafts through pages, rotary positions and attention: every token's
    result is that of attention over its whole text at once."""
    heads, kv, d, page, slots, td = 4, 2, 64, 16, 5, torch.bfloat16
    pool = M.CachePages.empty(slots, 60, 20)
    kc, vc = (torch.full((60, page, kv, d), float("nan"), device="cuda", dtype=td) for _ in range(2))
    freqs = M.rotary_frequencies(d)
    text = [[] for _ in range(slots)]  # (q, k, v) of each token kept, before rotation
    gen = torch.Generator(device="cuda").manual_seed(3)

    def call(which, new, kept=None, tree=None):
        n, m = sum(new), len(which)
        q, k, v = (torch.randn(n, h, d, device="cuda", generator=gen).to(td) for h in (heads, kv, kv))
        off, index = torch.tensor([0] + new, device="cuda").cumsum(0), _ints(which)
        place, position = (torch.empty(n, device="cuda", dtype=torch.int32) for _ in range(2))
        admitted = torch.empty(m, device="cuda", dtype=torch.int32)
        M.CachePages(tokens=n, seqs=m, slots=slots, page=page, pages=60, max_pages=20).run(
            None if kept is None else _ints(kept), *pool, place, position, admitted, offsets=off, slot_index=index)
        qr, o = torch.empty_like(q), torch.empty_like(q)
        M.Rotary(tokens=n, heads=heads, kv_heads=kv, dk=d, page=page, pages=60).run(q, k, v, position, freqs, qr, None, kc, vc, place)
        M.SoftmaxAttention(tokens=n, seqs=m, slots=slots, heads=heads, kv_heads=kv, dk=d, page=page, pages=60, max_pages=20,
                           mask="causal" if tree is None else "tree").run(
            qr, kc, vc, o, offsets=off, slot_index=admitted, lens=pool[0], table=pool[1], tree=tree)
        first = 0
        for i, (s, c) in enumerate(zip(which, new)):
            if kept is not None:
                text[s] = text[s][:kept[i]]
            base = len(text[s])
            text[s] += [(q[t], k[t], v[t]) for t in range(first, first + c)]
            if c:
                ks, vs = (torch.stack([x[a] for x in text[s]]) for a in (1, 2))
                pos = np.arange(base + c)
                f = freqs.cpu().numpy()
                kr = ref.rotary(_host(ks), pos, f, d, "half", 1.0)
                qh = ref.rotary(_host(q[first:first + c]), pos[base:], f, d, "half", 1.0)
                bits = None if tree is None else [x % (1 << 64) for x in tree[first:first + c].tolist()]
                on = ref.sees("causal" if tree is None else "tree", c, base + c, bits)
                want, w_abs, most = ref.softmax_attention(qh, kr, _host(vs), on, d ** -0.5)
                # turned q and k are rounded to bf16: scores are off by 2 r of their absolute sums, so weights are, twice in the quotient
                tol = ref.softmax_bound(want, w_abs, most, base + c, d, "bf16") + 2 * 2.1 * R * most[..., None] * w_abs
                assert (np.abs(_host(o[first:first + c]) - want) <= tol).all()
            first += c

    call([0, 3, 1], [70, 1, 33])
    for _ in range(3):
        call([1, 0, 3], [1, 1, 1])
    drafts = torch.tensor([1, 3, 5, 11], device="cuda").repeat(2)
    call([3, 0], [4, 4], tree=drafts)
    call([3, 0], [1, 1], kept=[5, 74])    # the first draft was right, the others go
    call([3, 0, 4], [0, 40, 100], kept=[0, 75, 0])
    call([3], [50])
