"""Softmax attention of few rows over keys of every kernel's head sizes, as they lie in memory (needs the GPU)."""
import pytest
import torch

from paper_2407_10730_amd import seqmix as M
from test_gpu_softmax import Soft, _gpu  # noqa: F401

pytestmark = pytest.mark.gpu


def _behind(p, value):
    """`value` in the rows of k and v behind the sequences' ends (packed: behind the last)."""
    for t in (p.k, p.v):
        if p.page:
            for i, (_, pages) in enumerate(p.where):
                if p.keys[i] % p.page:
                    t[int(pages[-1]), p.keys[i] % p.page:] = value
        else:
            row = t.stride(0)
            t.as_strided((row,), (1,), t.storage_offset() + t.shape[0] * row).fill_(value)


@pytest.mark.parametrize("page", (0, 16, 64))
@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("dv", (64, 128, 256))
@pytest.mark.parametrize("dk", (64, 128, 256))
def test_few_rows_of_every_head_size(dk, dv, dtype, page):
    """Rows in whole 16 bytes of each pair of the kernels' sizes, packed and in pages below and above a tile, many keys in parts
    and few whole; the keys end inside a tile, and nothing behind them counts."""
    for keys in ([301, 45], [2777, 1203], [30, 3]):
        p = Soft([1, 3], keys=keys, heads=4, kv_heads=2, dk=dk, dv=dv, dtype=dtype, page=page, mask="causal")
        assert p.op.plan().kernel == M.SEQMIX_KERNEL_STEP
        assert not page or (p.k.data_ptr() | p.v.data_ptr()) % 16 == 0
        _behind(p, float("nan"))
        p.run().check()


def _moved(t, by):
    """A copy of t with its strides, `by` elements further on from an address of 16 bytes."""
    last = sum((n - 1) * s for n, s in zip(t.shape, t.stride()))
    flat = torch.zeros(last + 1 + by + 16, dtype=t.dtype, device=t.device)
    assert flat.data_ptr() % 16 == 0
    return flat.as_strided(t.shape, t.stride(), by).copy_(t)


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("kw", [
    dict(new=[300]), dict(new=[1000, 90, 0, 3], heads=16, kv_heads=4), dict(new=[300, 7], keys=[2000, 900], page=16),
    dict(new=[130, 40], keys=[5000, 77], page=64, dk=128, dv=128), dict(new=[70, 150], keys=[333, 4000], mask="full", dk=256, dv=64),
    dict(new=[200], keys=[1300], dk=256, dv=256), dict(new=[24] * 3, keys=[3000, 24, 1900], mask="tree", heads=8, page=32),
    dict(new=[1] * 3, keys=[5000, 70, 900], page=16, heads=8), dict(new=[3, 1], keys=[90, 700], dk=96, dv=72),
    dict(new=[90], dk=72, dv=104, qscale=20.0), dict(new=[40] * 600, heads=2, kv_heads=1),
])
def test_results_do_not_depend_on_addresses(kw, dtype):
    """The same descriptor and numbers at addresses of 16 bytes and of one element give the same bits, also where values are not
    finite."""
    p = Soft(**dict(dict(heads=4, kv_heads=2, dk=64, dv=64, dtype=dtype), **kw))
    for bad in (False, True):
        if bad:
            p.v.view(-1, *p.v.shape[-2:])[9, 0, 5] = float("inf")
            p.k.view(-1, *p.k.shape[-2:])[20, -1, 3] = float("-inf")
        at = {n: getattr(p, n) for n in ("q", "k", "v")}
        outs = []
        for by in (0, 1, 3):
            for n, t in at.items():
                setattr(p, n, _moved(t, by))
            p.o = _moved(torch.full_like(at["q"][..., :1], 7).expand(p.o.shape).contiguous(), by)
            outs.append(p.run().o.clone())
        for n, t in at.items():
            setattr(p, n, t)
        for o in outs[1:]:
            same = (o == outs[0]) | (torch.isnan(o) & torch.isnan(outs[0]))
            assert same.all(), f"{int((~same).sum())} of {same.numel()} results differ"


@pytest.mark.parametrize("heads", (1, 3))
def test_more_workgroups_than_a_launch_holds(heads):
    """Single tokens that each see one key: as many workgroups, of 512 threads, as sequences times heads, past 2^32 threads (and, with 3
    heads, past 2^25 workgroups).  A row that sees one key is its value, bit by bit."""
    n = (1 << 23) + 1003 if heads == 1 else (1 << 25) // 3 + 1003
    q, k, v = (torch.randn(n, heads, 8, device="cuda", dtype=torch.bfloat16) for _ in range(3))
    o = torch.full_like(v, 7)
    op = M.SoftmaxAttention(tokens=n, seqs=n, heads=heads, dk=8)
    assert op.plan().kernel == M.SEQMIX_KERNEL_STEP and op.plan().shares == 0
    op.run(q, k, v, o)
    assert torch.equal(o, v)


def test_rotary_positions_of_more_tokens_than_a_launch_holds():
    """2^26 tokens and more, four to a workgroup of 256 threads: each launch's last and first tokens as calls of their own turn them."""
    n, part = (1 << 26) + 5003, 4096
    gen = torch.Generator("cuda").manual_seed(0)
    q, k, v = (torch.randn(n, 1, d, device="cuda", generator=gen).bfloat16() for d in (2, 4, 3))
    position = torch.arange(n, device="cuda", dtype=torch.int32) // 64
    place = torch.arange(n - 1, -1, -1, device="cuda", dtype=torch.int32)
    freqs = M.rotary_frequencies(2)
    pages = -(-n // 16)

    def call(at, qo, ko, kc, vc):
        m = q[at].shape[0]
        M.Rotary(tokens=m, heads=1, kv_heads=1, dk=2, dv=3, page=16, pages=pages, k_strides=(4, 2)).run(
            q[at], k[at][..., :2], v[at], position[at], freqs, qo, ko, kc, vc, place[at])

    def new(m):
        return torch.full((m, 1, 2), 7.0, device="cuda", dtype=q.dtype), torch.full((m, 1, 2), 7.0, device="cuda", dtype=q.dtype), \
            *(torch.full((pages, 16, 1, d), 7.0, device="cuda", dtype=q.dtype) for d in (2, 3))

    whole = new(n)
    call(slice(None), *whole)
    for first in (0, (1 << 25) - part // 2, (1 << 26) - part // 2, n - part):
        at = slice(first, first + part)
        want = new(part)
        call(at, *want)
        assert torch.equal(whole[0][at], want[0]) and torch.equal(whole[1][at], want[1])
        rows = place[at].long()
        for got, one in zip(whole[2:], want[2:]):
            assert torch.equal(got.flatten(0, 1)[rows], one.flatten(0, 1)[rows])
    assert not (whole[0] == 7).all(-1).any()


@pytest.mark.parametrize("new,keys", (([1] * 3, [5000, 70, 900]), ([300, 7], [2000, 900])))
def test_a_first_call_does_not_wait(new, keys):
    """A descriptor's first call, which allocates its workspace, returns while another stream has work queued; it and the next, on
    another stream, are right."""
    p, first = (Soft(new, keys=keys, heads=8, kv_heads=2, dk=128, dv=128, page=16) for _ in range(2))
    assert p.op.plan().workspace_bytes > 0
    first.run()  # (loads the kernels)
    want = first.o
    x = torch.randn(8192, 8192, device="cuda")
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        x @ x
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        y = x @ x
        for _ in range(40):
            torch.mm(x, x, out=y)
        done = side.record_event()
    p.run()
    assert not done.query(), "the call waited for another stream"
    assert torch.equal(p.o, want)
    p.o = torch.full_like(want, 7)
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(other):
        p.run()
    torch.cuda.synchronize()
    assert torch.equal(p.o, want)


def test_a_first_call_that_is_captured_in_a_reserved_workspace():
    """Without a call before it; eager calls and replays after it give the same, in either order."""
    for replay_first in (True, False):
        p = Soft([1] * 3, keys=[5000, 70, 900], heads=8, kv_heads=2, dk=128, dv=128, page=16)
        p.op.reserve()
        g, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side), torch.cuda.graph(g, stream=side):
            p.run()
        outs = []
        for replay in (replay_first, not replay_first) * 2:
            p.o.fill_(7)
            g.replay() if replay else p.run()
            outs.append(p.o.clone())
        p.check()
        assert all(torch.equal(o, outs[0]) for o in outs[1:])
