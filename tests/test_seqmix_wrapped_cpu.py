"""Tensors that have no memory of their own are refused by the helpers with an error, not by ending the process.

Fake tensors stand for ones on a GPU, so that the checks are the ones that a GPU's tensors pass; no call gets as far as a kernel.
"""
import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

from paper_2407_10730_amd import binding as B
from paper_2407_10730_amd import seqmix as M


@pytest.fixture
def norm(monkeypatch):
    """GateNorm.run(u, w, y=y) on fake tensors, without the look at the GPU's streams."""
    op = M.GateNorm(rows=4, width=8, dtype="f32")
    op._raw_stream = lambda dev: 0
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    with FakeTensorMode():
        yield op
    op.close()


def _fake(*shape, **kw):
    return torch.empty(*shape, device="cuda", **kw)


def _refused(f, text):
    with pytest.raises(B.Conv2dError, match=text) as e:
        f()
    assert e.value.status == B.CONV2D_E_INVALID


def test_fake_tensors(norm):
    _refused(lambda: norm.run(_fake(4, 8), _fake(8), y=_fake(4, 8)), "u has no memory")


@pytest.mark.parametrize("transform", ["vmap", "grad", "vjp", "functionalize"])
def test_transforms(norm, transform):
    w, y = _fake(8), _fake(4, 8)

    def f(u):
        norm.run(u, w, y=y)
        return u.sum()

    x = _fake(4, 8)
    call = {"vmap": lambda: torch.vmap(f)(_fake(3, 4, 8)), "grad": lambda: torch.func.grad(f)(x),
            "vjp": lambda: torch.func.vjp(f, x), "functionalize": lambda: torch.func.functionalize(f)(x)}[transform]
    _refused(call, "u has no memory")


def test_sparse_tensors(norm):
    _refused(lambda: norm.run(_fake(4, 8, layout=torch.sparse_coo), _fake(8), y=_fake(4, 8)), "sparse")


def test_negated_views(norm):
    _refused(lambda: norm.run(torch._neg_view(_fake(4, 8)), _fake(8), y=_fake(4, 8)), "negated")


def test_what_is_told_first(norm):
    _refused(lambda: norm.run(_fake(4, 9), _fake(8), y=_fake(4, 8)), r"u is \(4, 9\)")
    _refused(lambda: norm.run(_fake(8, 4).t(), _fake(8), y=_fake(4, 8)), "u has strides")
    _refused(lambda: norm.run(_fake(4, 8), torch.empty(8), y=_fake(4, 8)), "u has no memory")


def test_a_call_without_its_main_tensor(norm):
    conv = M.TokenConv(tokens=4, seqs=1, channels=8, width=3)
    attn = M.LinearAttention(tokens=4, seqs=1, heads=1, dk=8, dv=8)
    for name, call in (("u", lambda: norm.run(None, _fake(8), y=_fake(4, 8))), ("u", lambda: norm.run([1.0])),
                       ("y", lambda: conv.run(_fake(4, 8), None, None, None, None, None)),
                       ("o", lambda: attn.run(_fake(4, 1, 8), None, None, None, None, None, None))):
        with pytest.raises(TypeError, match=f"{name} is a tensor"):
            call()
