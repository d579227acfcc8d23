"""Attention's outputs within what each kernel's own roundings allow (needs the GPU).

`oracle.seqmix.attention_bound` derives the bound; beside it, point by point, each block of 16 tokens is held in the 2-norm:
a sum of roundings that are as often up as down stays below a bound that each point alone may reach.
"""
import numpy as np
import pytest
import torch

from oracle import seqmix as ref
from paper_2407_10730_amd import seqmix as M
from test_gpu_seqmix import Attn, _case, _gpu, _host, _near  # noqa: F401

pytestmark = pytest.mark.gpu


def _held(a, o_dtype):
    want, o_abs, _, _ = a.want()
    bound = ref.attention_bound(want, o_abs, max(a.lens), a.dk, a.dtype, o_dtype,
                                a.op.plan().kernel == M.SEQMIX_KERNEL_CHUNKS)
    got = _host(a.o)
    _near(got, want, bound + 1e-37, 1.0, "o")
    for first in range(0, len(want), 16):
        rows = slice(first, first + 16)
        off, most = np.linalg.norm(got[rows] - want[rows]), np.linalg.norm(bound[rows])
        assert off <= most, f"tokens from {first}: {off:.3g}, bound {most:.3g}"
    if o_dtype == "bf16" and a.dtype == "bf16":
        # one rounding to 8 bits is uniform over a unit in the last place: at most 2^-8 / sqrt(3) = 0.00226 in the
        # 2-norm (values at the low end of a binade)
        off = np.linalg.norm(got - want) / np.linalg.norm(want)
        print(f"  2-norm: {off:.5f}", flush=True)
        assert off <= 2.0 ** -8 / 3 ** 0.5


@pytest.mark.parametrize("kw", [
    *[_case(lens=[t], heads=2, qk_heads=1, dk=64, dv=64) for t in (3, 16, 17, 63, 64, 65, 90, 129)],
    *[_case(lens=[300], heads=2, qk_heads=2, dk=128, dv=128, decay=d) for d in ("token", "head", "none")],
    _case(lens=[260], heads=1, qk_heads=1, dk=256, dv=256),
    _case(lens=[260], heads=1, qk_heads=1, dk=200, dv=132),
    _case(lens=[130], heads=2, qk_heads=1, dk=33, dv=71),
    _case(lens=[2000], heads=1, qk_heads=1, dk=64, dv=96),
    _case(lens=[90] * 5, heads=2, qk_heads=1, dk=128, dv=128),
    _case(lens=[90] * 70, heads=8, qk_heads=2, dk=32, dv=128),
    _case(lens=[0, 70, 1, 0, 200, 64, 3, 900], heads=3, qk_heads=1, dk=64, dv=96),
    _case(lens=[1] * 3, heads=4, qk_heads=2, dk=128, dv=128),
    _case(lens=[2] * 2, heads=2, qk_heads=1, dk=256, dv=250),
])
@pytest.mark.parametrize("o_dtype", ["bf16", "f32"])
def test_attention_rounds_outputs_once(kw, o_dtype):
    print(f"\n[case] {kw} {o_dtype}", flush=True)
    a = Attn(**kw, o_dtype=o_dtype)
    a.run(a.state, torch.empty_like(a.state))
    _held(a, o_dtype)


@pytest.mark.parametrize("lens", [[65], [300], [1500]])
def test_attention_fp32_outputs_are_fp32_sums(lens):
    a = Attn(lens, 2, 1, 72, 40, dtype="f32")
    a.run(a.state, torch.empty_like(a.state))
    _held(a, "f32")


@pytest.mark.parametrize("lens", [[100], [2000]])
@pytest.mark.parametrize("o_dtype", ["bf16", "f32"])
@pytest.mark.parametrize("value", [float("inf"), -float("inf")])
def test_attention_takes_infinite_states(lens, o_dtype, value):
    """A state with an infinite column gives infinite outputs of that column, by the sign of q, as its definition does."""
    def edit(a):
        a.q.abs_().add_(0.01)

    a = Attn(lens, 1, 1, 64, 64, o_dtype=o_dtype, edit=edit)
    a.g.zero_()
    a.state[:, :, :, 5] = value
    a.run(a.state, torch.empty_like(a.state))
    got = _host(a.o)
    assert (got[:, :, 5] == value).all()
    assert np.isfinite(np.delete(got, 5, 2)).all()


def _set(a, first, start, v):
    """Log2 decays of `first` over the first segment and almost none after it; start states and values of size 2^start, 2^v."""
    seg = a.op.plan().segment
    assert a.op.plan().kernel == M.SEQMIX_KERNEL_CHUNKS and 0 < seg < a.lens[0] and abs(first) / seg * 64 < 100
    a.g.fill_(-0.001)
    a.g[:seg] = first / seg * float(np.log(2))
    a.state.mul_(2.0 ** start)
    a.v.mul_(2.0 ** v)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("first,start,v", [(150, -110, -110), (-150, 120, -30), (200, -110, -110), (-200, 120, -80)])
def test_attention_segments_grow_and_decay(dtype, first, start, v):
    """A segment's whole decay or growth may lie outside fp32 where what it is of, and what becomes of that, do not."""
    a = Attn([2000], 16, 16, 64, 64, dtype=dtype)
    if abs(first) == 200:
        a = Attn([8000], 16, 16, 64, 64, dtype=dtype)
    _set(a, first, start, v)
    left = torch.empty_like(a.state)
    a.run(a.state, left)
    _held(a, dtype)
    _, _, s, s_abs = a.want()
    _near(_host(left), s, s_abs, (2 * a.n + a.dk + 64) * 2.0 ** -24, "state")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("state", [True, False])
def test_attention_zeros_stay_zeros_under_growth(dtype, state):
    """Growth past every float of a state of zeros, for as long as keys and values are zeros."""
    a = Attn([2000], 16, 16, 64, 64, dtype=dtype, state=state)
    seg = a.op.plan().segment
    assert 0 < seg < 1000
    a.g[:1900] = 1.2 * float(np.log(2))
    assert 1.2 * seg > 128
    a.k[:1900] = 0.0
    a.v[:1900] = 0.0
    if state:
        a.state.zero_()
    left = torch.full((1, 16, 64, 64), 7.0, device="cuda")
    a.run(a.state, left)
    _held(a, dtype)
    assert not a.o[:1900].any()
    _, _, s, s_abs = a.want()
    _near(_host(left), s, s_abs, (2 * a.n + a.dk + 64) * 2.0 ** -24, "state")
