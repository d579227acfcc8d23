"""Softmax attention, rotary positions and cache pages on the CPU: refusals, the helpers' checks, the definitions themselves."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import seqmix as ref
from paper_2407_10730_amd import binding as B
from paper_2407_10730_amd import seqmix as M

INVALID, UNSUPPORTED, NULL = B.CONV2D_E_INVALID, B.CONV2D_E_UNSUPPORTED, B.CONV2D_E_NULL


def _soft(**kw):
    base = dict(tokens=10, seqs=2, slots=2, key_tokens=10, heads=4, kv_heads=2, dk=8, dv=16, dtype=B.CONV2D_BF16,
                mask=M.SEQMIX_MASK_CAUSAL, scale=1.0, q_row=32, q_head=8, o_row=64, o_head=16, k_row=16, k_head=8, v_row=32,
                v_head=16)
    base.update(kw)
    return M.seqmix_softmax_params(**base)


PAGED = dict(page=4, pages=6, max_pages=3, k_page=64, v_page=128)


@pytest.mark.parametrize("kw,code", [
    (dict(tokens=-1), INVALID), (dict(seqs=0), INVALID), (dict(slots=0), INVALID), (dict(heads=0), INVALID),
    (dict(kv_heads=3), INVALID), (dict(kv_heads=0), INVALID), (dict(dk=0), INVALID), (dict(dv=0), INVALID),
    (dict(q_row=31), INVALID), (dict(q_head=7), INVALID), (dict(o_head=-16), INVALID), (dict(k_row=15), INVALID),
    (dict(v_head=15), INVALID), (dict(scale=float("nan")), INVALID), (dict(scale=float("inf")), INVALID),
    (dict(key_tokens=-1), INVALID), (dict(mask=3), UNSUPPORTED), (dict(mask=-1), UNSUPPORTED), (dict(dtype=7), UNSUPPORTED),
    (dict(dk=257, q_row=1028, q_head=257, k_row=514, k_head=257), UNSUPPORTED),
    (dict(tokens=1 << 31), UNSUPPORTED), (dict(key_tokens=1 << 31), UNSUPPORTED),
    (dict(PAGED, page=3), INVALID), (dict(PAGED, page=-4), INVALID), (dict(PAGED, pages=0), INVALID),
    (dict(PAGED, max_pages=0), INVALID), (dict(PAGED, k_page=63), INVALID), (dict(PAGED, v_page=100), INVALID),
    (dict(PAGED, page=1 << 17), UNSUPPORTED), (dict(PAGED, pages=1 << 29), UNSUPPORTED),
    (dict(PAGED, max_pages=1 << 29), UNSUPPORTED),
    (dict(heads=1 << 21, kv_heads=1 << 21, q_row=1 << 24, o_row=1 << 25, k_row=1 << 24, v_row=1 << 25), UNSUPPORTED),
])
def test_softmax_refuses(kw, code):
    with pytest.raises(B.Conv2dError) as e:
        M.seqmix_softmax_desc_create(_soft(**kw))
    assert e.value.status == code


def _rotary(**kw):
    base = dict(tokens=10, page=4, pages=3, heads=4, kv_heads=2, dk=8, dv=16, rot=8, layout=0, dtype=1, amplitude=1.0, q_row=32,
                q_head=8, k_row=16, k_head=8, v_row=32, v_head=16, qo_row=32, qo_head=8, ko_row=16, ko_head=8, kc_row=16,
                kc_head=8, kc_page=64, vc_row=32, vc_head=16, vc_page=128)
    base.update(kw)
    return M.seqmix_rotary_params(**base)


@pytest.mark.parametrize("kw,code", [
    (dict(tokens=-1), INVALID), (dict(heads=-1), INVALID), (dict(kv_heads=-1), INVALID), (dict(dk=0), INVALID),
    (dict(rot=7), INVALID), (dict(rot=10), INVALID), (dict(rot=-2), INVALID), (dict(q_row=31), INVALID),
    (dict(qo_head=7), INVALID), (dict(ko_row=15), INVALID), (dict(v_row=31), INVALID), (dict(kv_heads=0), INVALID),
    (dict(dv=0), INVALID), (dict(page=6), INVALID), (dict(pages=0), INVALID), (dict(kc_page=60), INVALID),
    (dict(vc_row=30), INVALID), (dict(layout=2), UNSUPPORTED), (dict(dtype=2), UNSUPPORTED), (dict(tokens=1 << 31), UNSUPPORTED),
    (dict(dv=300, v_row=600, v_head=300, vc_row=600, vc_head=300, vc_page=2400), UNSUPPORTED),
    (dict(pages=1 << 29), UNSUPPORTED), (dict(page=1 << 17, kc_page=1 << 30, vc_page=1 << 30), UNSUPPORTED),
])
def test_rotary_refuses(kw, code):
    with pytest.raises(B.Conv2dError) as e:
        M.seqmix_rotary_desc_create(_rotary(**kw))
    assert e.value.status == code


@pytest.mark.parametrize("kw,code", [
    (dict(tokens=-1), INVALID), (dict(seqs=0), INVALID), (dict(slots=0), INVALID), (dict(page=0), INVALID),
    (dict(page=12), INVALID), (dict(pages=0), INVALID), (dict(max_pages=0), INVALID), (dict(tokens=1 << 31), UNSUPPORTED),
    (dict(pages=1 << 28), UNSUPPORTED), (dict(max_pages=1 << 28), UNSUPPORTED), (dict(page=1 << 20), UNSUPPORTED),
])
def test_pages_refuse(kw, code):
    with pytest.raises(B.Conv2dError) as e:
        M.seqmix_pages_desc_create(M.seqmix_pages_params(**dict(dict(tokens=4, seqs=2, slots=2, pages=5, max_pages=3, page=16), **kw)))
    assert e.value.status == code


def test_calls_refuse_missing_pointers_and_bad_packing():
    lib, one = M.load(), ctypes.c_void_p(64)
    for op in ("softmax", "rotary", "pages"):
        assert getattr(lib, f"seqmix_{op}_desc_create")(None, None) == NULL
        assert getattr(lib, f"seqmix_{op}_fwd")(*[None] * 12) == NULL
        assert getattr(lib, f"seqmix_{op}_desc_destroy")(None) == B.CONV2D_OK
    assert lib.seqmix_softmax_plan_query(None, None) == NULL
    assert lib.seqmix_softmax_reserve(None) == NULL

    def missing(fn, desc, full, places, code=NULL):
        for at in places:
            args = list(full)
            args[at] = None
            assert fn(desc, *args, None) == code, at

    # q, k, v, offsets, key_offsets, slot_index, lens, table, tree, o
    full = [one] * 10
    d = M.seqmix_softmax_desc_create(_soft(mask=M.SEQMIX_MASK_TREE))
    missing(lib.seqmix_softmax_fwd, d, full, (0, 1, 2, 8, 9))
    M.seqmix_softmax_desc_destroy(d)
    d = M.seqmix_softmax_desc_create(_soft(**PAGED))
    missing(lib.seqmix_softmax_fwd, d, full, (0, 1, 2, 6, 7, 9))
    M.seqmix_softmax_desc_destroy(d)
    d = M.seqmix_softmax_desc_create(_soft(tokens=11, slots=1))
    missing(lib.seqmix_softmax_fwd, d, full, (3, 5), INVALID)     # 11 rows in 2 sequences; 1 slot
    missing(lib.seqmix_softmax_fwd, d, full[:5] + [one] + full[6:], (4,), INVALID)  # 10 keys and 11 rows
    M.seqmix_softmax_desc_destroy(d)
    d = M.seqmix_softmax_desc_create(_soft(tokens=0, key_tokens=0))
    assert lib.seqmix_softmax_fwd(d, *[None] * 11) == B.CONV2D_OK  # nothing to do
    M.seqmix_softmax_desc_destroy(d)

    # q, k, v, position, freqs, q_out, k_out, k_cache, v_cache, place
    d = M.seqmix_rotary_desc_create(_rotary())
    missing(lib.seqmix_rotary_fwd, d, full, (0, 1, 2, 3, 4, 5, 7, 8, 9))
    M.seqmix_rotary_desc_destroy(d)

    # kept, offsets, slot_index, lens, table, free_pages, taken, place, position, admitted
    d = M.seqmix_pages_desc_create(M.seqmix_pages_params(tokens=5, seqs=2, slots=1, pages=5, max_pages=3, page=16))
    missing(lib.seqmix_pages_fwd, d, full, (3, 4, 5, 6, 7, 8, 9))
    missing(lib.seqmix_pages_fwd, d, full, (1, 2), INVALID)
    M.seqmix_pages_desc_destroy(d)


def test_helpers_refuse():
    for make in (lambda: M.SoftmaxAttention(tokens=4, seqs=1, heads=1, dk=8, mask="window"),
                 lambda: M.SoftmaxAttention(tokens=4, seqs=1, heads=1, dk=8, dtype="f16"),
                 lambda: M.Rotary(tokens=4, heads=1, kv_heads=1, dk=8, layout="whole"),
                 lambda: M.rotary_frequencies(8, factor=2.0, trained=100, low=4.0, high=4.0, device="cpu")):
        with pytest.raises(ValueError):
            make()
    op = M.SoftmaxAttention(tokens=4, seqs=1, heads=2, dk=8, dtype="f32")
    x = torch.zeros(4, 2, 8)
    for bad in (torch.zeros(4, 2, 9), x.bfloat16(), torch.zeros(2, 4, 8).transpose(0, 1), x):  # the last: not on a GPU
        with pytest.raises(B.Conv2dError) as e:
            op.run(bad, x, x, x)
        assert e.value.status == INVALID
    with pytest.raises(TypeError):
        op.run(x, x, x, None)
    with pytest.raises(B.Conv2dError):  # tables are those of the pool
        M.SoftmaxAttention(tokens=1, seqs=1, heads=1, dk=8, page=16, pages=4, max_pages=2).run(
            x, x, x, x, lens=torch.zeros(1, dtype=torch.int32), table=torch.zeros(2, 2, dtype=torch.int32))
    op = M.Rotary(tokens=4, heads=2, kv_heads=2, dk=8, dtype="f32")
    with pytest.raises(B.Conv2dError):  # frequencies are float64
        op.run(x, x, None, torch.zeros(4, dtype=torch.int32), torch.zeros(4), x, x)
    op = M.CachePages(tokens=4, seqs=1, page=16, pages=4, max_pages=2)
    pool = M.CachePages.empty(1, 4, 2, device="cpu")
    with pytest.raises(B.Conv2dError):
        op.run(None, *pool, *(torch.zeros(n, dtype=torch.int32) for n in (4, 4, 1)))


def test_plans_of_prompts_and_single_tokens():
    def plan(**kw):
        return M.SoftmaxAttention(**dict(dict(heads=16, kv_heads=4, dk=128), **kw)).plan()
    assert plan(tokens=8192, seqs=1).pack == 1
    assert plan(tokens=64, seqs=64, page=16, pages=100, max_pages=50).pack == 4
    assert plan(tokens=64, seqs=64, heads=60, kv_heads=5, page=16, pages=100, max_pages=50).pack == 12


def test_frequencies():
    f = M.rotary_frequencies(64, base=500000.0, device="cpu")
    assert f.dtype == torch.float64 and np.allclose(f.numpy(), 500000.0 ** (-np.arange(32) / 32), rtol=1e-14)
    assert torch.equal(M.rotary_frequencies(64, base=500000.0, factor=8.0, device="cpu"), f / 8)
    g = M.rotary_frequencies(64, base=500000.0, factor=8.0, trained=8192, device="cpu")
    turns = 8192 * f / (2 * np.pi)
    assert torch.equal(g[turns > 4], f[turns > 4]) and torch.allclose(g[turns < 1], f[turns < 1] / 8, rtol=1e-15)
    between = (turns > 1) & (turns < 4)
    assert between.any() and (g[between] < f[between]).all() and (g[between] > f[between] / 8).all()


def test_definitions():
    """The float64 definitions against torch's, and what masks mean."""
    rng = np.random.default_rng(0)
    q, k, v = (torch.from_numpy(rng.standard_normal((n, h, d))) for n, h, d in ((5, 4, 8), (9, 2, 8), (9, 2, 6)))
    on = ref.sees("causal", 5, 9)
    assert on[0].tolist() == [True] * 5 + [False] * 4 and on[4].all()
    o, o_abs, most = ref.softmax_attention(q.numpy(), k.numpy(), v.numpy(), on, 0.3)
    kk, vv = (x.repeat_interleave(2, 1).transpose(0, 1) for x in (k, v))
    s = (q.transpose(0, 1) @ kk.transpose(1, 2) * 0.3).masked_fill(~torch.from_numpy(on), float("-inf"))
    assert np.allclose(o, (s.softmax(-1) @ vv).transpose(0, 1).numpy(), rtol=1e-12)
    assert (o_abs >= np.abs(o) - 1e-12).all()
    assert (most >= s.masked_fill(torch.isinf(s), 0).abs().amax(-1).t().numpy()).all()
    assert not ref.sees("causal", 4, 2)[:2].any() and ref.sees("causal", 4, 2)[3].all()
    tree = ref.sees("tree", 3, 5, [1, 3, 4])
    assert tree.tolist() == [[1, 1, 1, 0, 0], [1, 1, 1, 1, 0], [1, 1, 0, 0, 1]]
    x = rng.standard_normal((3, 2, 6))
    f = np.array([1.0, 0.25])
    y = ref.rotary(x, np.array([0, 2, 5]), f, 4, "interleaved", 1.0)
    assert np.array_equal(y[0], x[0]) and np.array_equal(y[..., 4:], x[..., 4:])
    z = (x[1, 0, 0] + 1j * x[1, 0, 1]) * np.exp(2j)
    assert np.allclose(y[1, 0, :2], [z.real, z.imag])
