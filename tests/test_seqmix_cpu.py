"""The token-mixing ABI on the CPU: exports, refusals, and the checks of the device-side helpers."""
import ctypes
import os
import re
import subprocess

import pytest
import torch

from paper_2407_10730_amd import binding as B
from paper_2407_10730_amd import seqmix as M

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_library_exports_every_declared_function():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "seqmix.h")).read(), flags=re.S)
    decl = set(re.findall(r"^\s*int\s+(seqmix_\w+)\s*\(", text, flags=re.M))
    assert decl == set(M.EXPORTS)
    out = subprocess.run(["nm", "-D", "--defined-only", B.LIB_PATH], capture_output=True, text=True, check=True).stdout
    assert decl <= set(re.findall(r"\bT (seqmix_\w+)", out))
    M.load()


def _attn(**kw):
    base = dict(tokens=10, seqs=2, slots=2, heads=4, qk_heads=2, dk=8, dv=16, dtype=B.CONV2D_BF16,
                o_dtype=B.CONV2D_BF16, decay=M.SEQMIX_DECAY_TOKEN, scale=1.0, q_row=16, q_head=8, k_row=16, k_head=8,
                v_row=64, v_head=16, o_row=64, o_head=16)
    base.update(kw)
    return M.seqmix_attn_params(**base)


@pytest.mark.parametrize("kw,code", [
    (dict(tokens=-1), B.CONV2D_E_INVALID), (dict(seqs=0), B.CONV2D_E_INVALID), (dict(slots=0), B.CONV2D_E_INVALID),
    (dict(heads=0), B.CONV2D_E_INVALID), (dict(qk_heads=3), B.CONV2D_E_INVALID), (dict(dk=0), B.CONV2D_E_INVALID),
    (dict(dv=0), B.CONV2D_E_INVALID), (dict(decay=3), B.CONV2D_E_INVALID), (dict(q_row=15), B.CONV2D_E_INVALID),
    (dict(k_head=7), B.CONV2D_E_INVALID), (dict(v_row=0), B.CONV2D_E_INVALID), (dict(o_head=-16), B.CONV2D_E_INVALID),
    (dict(dk=257, q_row=514, q_head=257, k_row=514, k_head=257), B.CONV2D_E_UNSUPPORTED),
    (dict(dtype=7), B.CONV2D_E_UNSUPPORTED), (dict(dtype=B.CONV2D_F32), B.CONV2D_E_UNSUPPORTED),
    (dict(tokens=1 << 31, seqs=1), B.CONV2D_E_UNSUPPORTED),
])
def test_attention_refuses(kw, code):
    with pytest.raises(B.Conv2dError) as e:
        M.seqmix_attn_desc_create(_attn(**kw))
    assert e.value.status == code


def test_attention_takes_heads_outside_rows():
    """[heads][tokens][d] memory is as good as [tokens][heads][d]."""
    d = M.seqmix_attn_desc_create(_attn(q_row=8, q_head=80, v_row=16, v_head=160))
    M.seqmix_attn_desc_destroy(d)
    with pytest.raises(B.Conv2dError):  # heads that overlap
        M.seqmix_attn_desc_create(_attn(q_row=8, q_head=72))


@pytest.mark.parametrize("kw,code", [
    (dict(tokens=-1), B.CONV2D_E_INVALID), (dict(channels=0), B.CONV2D_E_INVALID), (dict(width=0), B.CONV2D_E_INVALID),
    (dict(x_row=31), B.CONV2D_E_INVALID), (dict(y_row=31), B.CONV2D_E_INVALID),
    (dict(width=9), B.CONV2D_E_UNSUPPORTED), (dict(dtype=2), B.CONV2D_E_UNSUPPORTED),
    (dict(act=M.SEQMIX_ACT_SIGMOID), B.CONV2D_E_UNSUPPORTED),
    (dict(channels=(1 << 31) - 1, x_row=1 << 31, y_row=1 << 31), B.CONV2D_E_UNSUPPORTED),
])
def test_convolution_refuses(kw, code):
    base = dict(tokens=6, seqs=2, slots=2, channels=32, width=4, dtype=0, act=1, has_bias=1, x_row=32, y_row=32)
    base.update(kw)
    with pytest.raises(B.Conv2dError) as e:
        M.seqmix_conv_desc_create(M.seqmix_conv_params(**base))
    assert e.value.status == code


@pytest.mark.parametrize("kw,code", [
    (dict(rows=-1), B.CONV2D_E_INVALID), (dict(width=0), B.CONV2D_E_INVALID), (dict(group=7), B.CONV2D_E_INVALID),
    (dict(gate_run=0), B.CONV2D_E_INVALID), (dict(post_eps=-1.0), B.CONV2D_E_INVALID),
    (dict(pre_eps=float("nan")), B.CONV2D_E_INVALID), (dict(u_row=63), B.CONV2D_E_INVALID),
    (dict(gate=1, gate_row=63), B.CONV2D_E_INVALID), (dict(h_row=0), B.CONV2D_E_INVALID),
    (dict(group=32), B.CONV2D_E_UNSUPPORTED),  # pre norms whole rows
    (dict(post=3), B.CONV2D_E_UNSUPPORTED), (dict(pre=-1), B.CONV2D_E_UNSUPPORTED),
    (dict(gate=4), B.CONV2D_E_UNSUPPORTED), (dict(dtype=0, res_dtype=1), B.CONV2D_E_UNSUPPORTED),
    (dict(width=16392, group=16392, u_row=16392, res_row=16392, y_row=16392, h_row=16392), B.CONV2D_E_UNSUPPORTED),
])
def test_norm_refuses(kw, code):
    base = dict(rows=4, width=64, group=64, gate_run=1, dtype=1, res_dtype=1, post=1, pre=2, residual=1, scale=1.0,
                u_row=64, gate_row=64, res_row=64, y_row=64, h_row=64)
    base.update(kw)
    with pytest.raises(B.Conv2dError) as e:
        M.seqmix_norm_desc_create(M.seqmix_norm_params(**base))
    assert e.value.status == code


def test_calls_refuse_missing_pointers_and_bad_packing():
    lib, one = M.load(), ctypes.c_void_p(64)
    assert lib.seqmix_attn_desc_create(None, None) == B.CONV2D_E_NULL
    assert lib.seqmix_attn_fwd(*[None] * 11) == B.CONV2D_E_NULL
    assert lib.seqmix_conv_fwd(*[None] * 10) == B.CONV2D_E_NULL
    assert lib.seqmix_norm_fwd(*[None] * 12) == B.CONV2D_E_NULL
    assert lib.seqmix_attn_plan_query(None, None) == B.CONV2D_E_NULL
    assert lib.seqmix_attn_reserve(None) == B.CONV2D_E_NULL
    for destroy in (lib.seqmix_attn_desc_destroy, lib.seqmix_conv_desc_destroy, lib.seqmix_norm_desc_destroy):
        assert destroy(None) == B.CONV2D_OK
    a = M.seqmix_attn_desc_create(_attn(tokens=11, slots=1))
    full = [a, one, one, one, one, one, one, one, one, one, None]
    for missing in (1, 2, 3, 4, 9):
        args = list(full)
        args[missing] = None
        assert lib.seqmix_attn_fwd(*args) == B.CONV2D_E_NULL
    assert lib.seqmix_attn_fwd(a, one, one, one, one, None, one, one, one, one, None) == B.CONV2D_E_INVALID  # 11 / 2
    assert lib.seqmix_attn_fwd(a, one, one, one, one, one, None, one, one, one, None) == B.CONV2D_E_INVALID  # 1 slot
    M.seqmix_attn_desc_destroy(a)
    n = M.seqmix_norm_desc_create(M.seqmix_norm_params(
        rows=4, width=64, group=64, gate_run=1, dtype=1, res_dtype=1, post=1, pre=1, residual=1, scale=1.0, u_row=64,
        res_row=64, y_row=64, h_row=64))
    args = [n, one, one, None, None, one, None, one, None, one, one, None]
    assert lib.seqmix_norm_fwd(*args) == B.CONV2D_E_INVALID  # h is y
    for missing in (1, 2, 5, 7, 10):
        bad = list(args)
        bad[missing] = None
        assert lib.seqmix_norm_fwd(*bad) == B.CONV2D_E_NULL
    M.seqmix_norm_desc_destroy(n)


def _plan(**kw):
    d = M.seqmix_attn_desc_create(_attn(**kw))
    p = M.seqmix_attn_plan_query(d)
    M.seqmix_attn_desc_destroy(d)
    return p


def test_attention_plans():
    dims = dict(dk=128, dv=128, heads=8, qk_heads=8, q_row=1024, q_head=128, k_row=1024, k_head=128, v_row=1024,
                v_head=128, o_row=1024, o_head=128)
    one = _plan(tokens=64, seqs=64, slots=64, **dims)
    assert (one.kernel, one.segment, one.workspace_bytes) == (M.SEQMIX_KERNEL_TOKENS, 0, 0)
    assert _plan(tokens=5 * 64, seqs=64, slots=64, **dims).kernel == M.SEQMIX_KERNEL_CHUNKS
    assert _plan(tokens=300, seqs=1, slots=1, **dims).segment == 0        # a few chunks: not worth a second pass
    assert _plan(tokens=1 << 16, seqs=64, slots=64, **dims).segment == 0  # enough sequences side by side
    cut = _plan(tokens=1 << 16, seqs=1, slots=1, **dims)
    assert cut.segment % cut.chunk == 0 and 0 < cut.segment < 1 << 16
    assert cut.workspace_bytes >= (1 << 16) // cut.segment * 8 * 128 * 128 * 4
    # rows too far apart for the chunk kernels' 32-bit offsets
    assert _plan(tokens=1 << 10, seqs=1, slots=1, **dict(dims, q_row=1 << 24)).kernel == M.SEQMIX_KERNEL_TOKENS


def test_helpers_refuse_tensors_that_do_not_fit():
    op = M.TokenConv(tokens=4, seqs=1, channels=8, width=3, dtype="f32")
    x = torch.zeros(4, 8)
    ok = (x, torch.zeros(8, 3), torch.zeros(8), None, None, torch.zeros(4, 8))
    for at, bad in ((0, torch.zeros(4, 9)), (0, x.bfloat16()), (0, torch.zeros(8, 4).t()), (1, torch.zeros(3, 8)),
                    (5, torch.zeros(5, 8)), (0, x)):  # the last: not on a GPU
        args = list(ok)
        args[at] = bad
        with pytest.raises(B.Conv2dError) as e:
            op.run(*args)
        assert e.value.status == B.CONV2D_E_INVALID
    with pytest.raises(TypeError):
        op.run(x.tolist(), *ok[1:])
    op.close()
    for make in (lambda: M.TokenConv(tokens=4, seqs=1, channels=8, width=3, dtype="f16"),
                 lambda: M.TokenConv(tokens=4, seqs=1, channels=8, width=3, act="relu"),
                 lambda: M.LinearAttention(tokens=4, seqs=1, heads=1, dk=8, dv=8, decay="row"),
                 lambda: M.GateNorm(rows=4, width=8, post="batch")):
        with pytest.raises(ValueError):
            make()
