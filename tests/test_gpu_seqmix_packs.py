"""Packs of very unequal sequences, and long ones (needs the GPU)."""
import numpy as np
import pytest
import torch

from test_gpu_seqmix import Attn, _gpu, _host, _near  # noqa: F401
from test_gpu_seqmix_bounds import _held

pytestmark = pytest.mark.gpu


def _check(a):
    left, other = a.state.clone(), np.setdiff1d(np.arange(a.slots), a.index)
    a.run(left, left)
    _held(a, a.dtype)
    _, _, s, s_abs = a.want()
    _near(_host(left)[a.index], s, s_abs, (2 * max(a.lens) + a.dk + 64) * 2.0 ** -24, "state")
    assert torch.equal(left[other], a.state[other])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens,heads", [
    ([100] * 20 + [3000] + [100] * 19, 16),    # enough sequences for the card, one of them long
    ([70] * 31 + [2000], 16),
    ([0] * 100 + [512] + [0] * 155, 2),        # empty places and one prompt, under two tokens on average
    ([1] * 200 + [257] + [1] * 55, 2),         # single tokens and one prompt, two on average
    ([1] * 60 + [0] * 300 + [900] + [2] * 40, 1),
], ids=lambda x: f"{len(x)}-{sum(x)}" if isinstance(x, list) else str(x))
def test_one_long_sequence_among_many(dtype, lens, heads):
    _check(Attn(lens, heads, heads, 32, 40, dtype=dtype, pool=2, uniform=False))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens", [[30011], [20000, 3, 7001]], ids=str)
def test_tens_of_thousands_of_tokens(dtype, lens):
    a = Attn(lens, 1, 1, 32, 24, dtype=dtype, pool=1, uniform=False)
    assert a.op.plan().segment > 0
    _check(a)
