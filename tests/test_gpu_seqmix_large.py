"""Token-mixing calls of more threads than a launch holds (needs the GPU)."""
import pytest
import torch

from paper_2407_10730_amd import seqmix as M

pytestmark = pytest.mark.gpu


def test_norm():
    """Sixteen rows to a workgroup of 256 threads: rows before and behind 2^32 threads are as in calls of their own."""
    edge, part = 1 << 28, 4096
    rows = edge + 5003
    u = torch.randn(rows, 3, device="cuda", dtype=torch.bfloat16)
    w = torch.rand(3, device="cuda") + 0.5
    y = torch.full_like(u, 7)
    M.GateNorm(rows=rows, width=3).run(u, w, y=y)
    op, one = M.GateNorm(rows=part, width=3), torch.empty(part, 3, device="cuda", dtype=u.dtype)
    for first in (0, edge - part // 2, rows - part):
        op.run(u[first:first + part], w, y=one)
        assert torch.equal(y[first:first + part], one)
    assert not (y == 7).any()


def test_linear_attention():
    """A workgroup of 256 threads to a single token and head: tokens before and behind 2^32 threads are as in calls of their own."""
    n, part = (1 << 24) + 5003, 4096
    q, k, v = (torch.randn(n, 1, d, device="cuda", dtype=torch.bfloat16) for d in (2, 2, 3))
    state, o = torch.randn(n, 1, 2, 3, device="cuda"), torch.full_like(v, 7)
    left = torch.full_like(state, 7)
    op = M.LinearAttention(tokens=n, seqs=n, heads=1, dk=2, dv=3, decay="none")
    assert op.plan().kernel == M.SEQMIX_KERNEL_TOKENS
    op.run(q, k, v, None, state, left, o)
    op, o1, left1 = M.LinearAttention(tokens=part, seqs=part, heads=1, dk=2, dv=3, decay="none"), o[:part].clone(), left[:part].clone()
    for first in (0, (1 << 24) - part // 2, n - part):
        at = slice(first, first + part)
        op.run(q[at], k[at], v[at], None, state[at], left1, o1)
        assert torch.equal(o[at], o1) and torch.equal(left[at], left1)
