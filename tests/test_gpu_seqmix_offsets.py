"""Offsets that lie, where sequences are searched for and cut: wrong results, but no access outside the tensors (needs the GPU)."""
import numpy as np
import pytest
import torch

from paper_2407_10730_amd import seqmix as M
from test_gpu_seqmix import Attn, _gpu  # noqa: F401
from test_gpu_seqmix_packs import _check

pytestmark = pytest.mark.gpu


def _lies(n):
    """For four sequences: not ascending, out of range, and first ones above 0, below which no sequence is found."""
    big = 1 << 40
    return ([0, n, n, n, n], [0, big, 0, big, n], [n, 0, n, 0, n], [-big, big, -big, big, -big], [900, 100, 2000, 3, 1],
            [0, 1500, 700, 2200, 100], [n - 1, n - 1000, n, n - 1500, n], [big] * 5, [-1] * 5, [0] * 5, [0, 0, 0, 0, n],
            [n // 2, n // 2, n, n, n])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_offsets_that_lie_where_sequences_are_cut(dtype):
    """Wrong results, but nothing outside the tensors is written, and the next call is right."""
    lens = [1500, 0, 800, 1]
    a = Attn(lens, 2, 2, 64, 96, dtype=dtype, uniform=False, pool=3)
    assert a.op.plan().segment > 0
    n, right = a.n, a.off_t
    home = torch.full((n + 128, 2, 96), 5.0, device="cuda").to(a.o.dtype)
    pool = torch.full((a.slots + 2, 2, 64, 96), 3.0, device="cuda")
    o, left = home[64:-64], pool[1:-1]
    for off in _lies(n):
        print(f"  {off}", flush=True)
        left.copy_(a.state)
        a.op.run(a.q, a.k, a.v, a.g, left, left, o, offsets=torch.tensor(off, device="cuda"), slot_index=a.slot_t)
        torch.cuda.synchronize()
        assert bool((home[:64] == 5.0).all()) and bool((home[-64:] == 5.0).all())
        assert bool((pool[0] == 3.0).all()) and bool((pool[-1] == 3.0).all())
        other = np.setdiff1d(np.arange(a.slots), a.index)
        assert torch.equal(left[other], a.state[other])
    a.off_t = right
    _check(a)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_convolution_offsets_that_lie(dtype):
    lens, c = [1500, 0, 800, 1], 72
    n, td = sum(lens), torch.float32 if dtype == "f32" else torch.bfloat16
    op = M.TokenConv(tokens=n, seqs=4, slots=6, channels=c, width=4, dtype=dtype)
    x, w, b = torch.randn(n, c, device="cuda").to(td), torch.randn(c, 4, device="cuda").to(td), torch.randn(c, device="cuda")
    slots = torch.tensor([4, 0, 5, 2], dtype=torch.int32, device="cuda")
    home, pool = torch.full((n + 128, c), 5.0, device="cuda").to(td), torch.full((8, 3, c), 3.0, device="cuda").to(td)
    y, win = home[64:-64], pool[1:-1]
    before = torch.randn(6, 3, c, device="cuda").to(td)

    def run(off):
        win.copy_(before)
        op.run(x, w, b, win, win, y, offsets=torch.tensor(off, device="cuda"), slot_index=slots)
        torch.cuda.synchronize()
        return y.clone(), win.clone()

    right = [0, *np.cumsum(lens).tolist()]
    want = run(right)
    for off in _lies(n):
        print(f"  {off}", flush=True)
        run(off)
        assert bool((home[:64] == 5.0).all()) and bool((home[-64:] == 5.0).all())
        assert bool((pool[0] == 3.0).all()) and bool((pool[-1] == 3.0).all())
        assert torch.equal(win[[1, 3]], before[[1, 3]])
    assert all(torch.equal(g, t) for g, t in zip(run(right), want))
