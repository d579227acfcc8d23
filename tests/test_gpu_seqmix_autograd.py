"""The token-mixing helpers beside autograd (needs the GPU): they are forward operators and say so."""
import pytest
import torch

from paper_2407_10730_amd import binding as B
from paper_2407_10730_amd import seqmix as M

pytestmark = pytest.mark.gpu


def _norm():
    op = M.GateNorm(rows=4, width=8, dtype="f32", gate="silu", residual=True, scale_vec=True, pre="layer", pre_bias=True,
                    post_bias=True, post="layer")
    t = {n: torch.rand(4, 8, device="cuda") for n in ("u", "gate", "residual", "y", "h")}
    t.update({n: torch.rand(8, device="cuda") for n in ("post_w", "post_b", "scale_vec", "pre_w", "pre_b")})
    return op, t, ("y", "h")


def _conv():
    op = M.TokenConv(tokens=4, seqs=1, channels=8, width=3, dtype="f32")
    t = {n: torch.rand(4, 8, device="cuda") for n in ("x", "y")}
    t.update({n: torch.rand(1, 2, 8, device="cuda") for n in ("window_in", "window_out")})
    return op, dict(t, w=torch.rand(8, 3, device="cuda"), bias=torch.rand(8, device="cuda")), ("y", "window_out")


def _attn():
    op = M.LinearAttention(tokens=4, seqs=1, heads=1, dk=8, dv=8, dtype="f32")
    t = {n: torch.rand(4, 1, 8, device="cuda") for n in "qkvo"}
    t.update({n: torch.rand(1, 1, 8, 8, device="cuda") for n in ("state_in", "state_out")})
    return op, dict(t, decay=-torch.rand(4, 1, device="cuda")), ("o", "state_out")


@pytest.mark.parametrize("make", [_norm, _conv, _attn])
def test_gradients_are_not_cut_off_silently(make):
    op, t, _ = make()
    op.run(**t)
    for name in t:
        with_grad = dict(t, **{name: t[name].clone().requires_grad_()})
        with pytest.raises(B.Conv2dError, match=f"{name} requires a gradient") as e:
            op.run(**with_grad)
        assert e.value.status == B.CONV2D_E_INVALID
        with torch.no_grad():
            op.run(**with_grad)
        with torch.inference_mode():
            op.run(**with_grad)


@pytest.mark.parametrize("make", [_norm, _conv, _attn])
def test_outputs_count_as_written(make):
    """A graph that holds an output's former values does not compute gradients with the new ones."""
    op, t, outs = make()
    for name in outs:
        w = torch.ones_like(t[name], requires_grad=True)
        y = (w * t[name]).sum()
        op.run(**t)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.backward()
    versions = {n: x._version for n, x in t.items()}
    op.run(**t)
    assert {n for n, x in t.items() if x._version != versions[n]} == set(outs)


def test_inference_tensors():
    with torch.inference_mode():
        op, t, _ = _norm()
        op.run(**t)
    op.run(**t)
