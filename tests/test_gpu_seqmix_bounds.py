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
