"""Softmax attention over values that are infinite or NaN, where the rows' maxima move far (needs the GPU)."""
import numpy as np
import pytest
import torch

from oracle import seqmix as ref
from paper_2407_10730_amd import seqmix as M
from test_gpu_softmax import Soft, _gpu, _host  # noqa: F401

pytestmark = pytest.mark.gpu

STEP, PROMPT = M.SEQMIX_KERNEL_STEP, M.SEQMIX_KERNEL_PROMPT


def _rising(p, gap, every):
    """Scores that rise by `gap` every so many keys, whatever block, share or wave a key falls to."""
    p.q[..., 0] = 1
    for i in range(len(p.new)):
        rise = gap * (torch.arange(p.keys[i], device="cuda") // every)
        first = sum(p.keys[:i])
        p.k[first:first + p.keys[i], :, 0] = rise.to(p.k.dtype)[:, None]


@pytest.mark.parametrize("gap", (200, 1000))
@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("kernel,new,keys,heads,kv_heads,dk,dv,shared", [
    (PROMPT, 40, 300, 2, 1, 64, 64, None),           # (fp32 is divided here, bf16 is not)
    (PROMPT, 150, 1500, 4, 2, 64, 96, True),
    (PROMPT, 33, 300, 520, 520, 64, 64, False),
    (PROMPT, 40, 300, 2, 1, 67, 71, None),
    (PROMPT, 150, 1500, 2, 1, 200, 256, True),
    (STEP, 3, 700, 4, 2, 64, 64, None),
    (STEP, 1, 5000, 4, 1, 128, 128, True),
    (STEP, 2, 700, 1030, 1030, 64, 64, False),
    (STEP, 3, 5000, 2, 2, 99, 130, True),
])
def test_values_before_far_higher_scores(kernel, new, keys, heads, kv_heads, dk, dv, shared, dtype, gap):
    """A row that sees a value that is not finite is NaN there, however much higher the scores of later keys are; no other
    result is touched."""
    p = Soft([new], keys=[keys], heads=heads, kv_heads=kv_heads, dk=dk, dv=dv, dtype=dtype, scale=1.0, qscale=0.1)
    plan = p.op.plan()
    assert plan.kernel == kernel and (shared is None or (plan.shares > 0) == shared)
    _rising(p, gap, 64)
    p.v[3, 0, 5], p.v[4, kv_heads - 1, 7], p.v[70, 0, 9] = float("inf"), float("nan"), float("-inf")
    p.v[keys - 1, 0, 11] = float("nan")  # seen by the last row only
    got, q = _host(p.run().o), _host(p.q)
    k, v = p.held(0)
    on = ref.sees("causal", new, keys)
    o, o_abs, most = ref.softmax_attention(q, k, v, on, p.scale)
    fine = np.isfinite(o)
    rep = heads // kv_heads
    want = np.zeros(o.shape, bool)
    want[:, :rep, [5, 9]] = True
    want[:, -rep:, 7] = True
    want[-1, :rep, 11] = True
    assert np.array_equal(~fine, want)
    assert np.array_equal(np.isnan(got), want) and np.isfinite(got[fine]).all()
    bound = ref.softmax_bound(o, o_abs, most, keys, dk, dtype, p.parts())
    assert (np.abs(got - o)[fine] <= bound[fine]).all()


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("new,heads,kv_heads,keys", [([70] * 2, 4, 4, 6000), ([1] * 16, 8, 8, 3000)])
def test_places_without_a_row_cost_nothing(new, heads, kv_heads, keys, dtype):
    """Keys of -infinity that every row gives a weight of zero: no pass over the keys is done again for the places of a tile
    that no row has (their scores are not numbers)."""
    p = Soft(new, keys=[keys] * len(new), heads=heads, kv_heads=kv_heads, dk=128, dv=128, dtype=dtype)
    p.q[..., 0] = 1

    def timed(value):
        p.k[5::100, :, 0] = value
        best = []
        for _ in range(6):
            a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            a.record()
            for _ in range(20):
                p.run()
            b.record()
            b.synchronize()
            best.append(a.elapsed_time(b))
        return min(best), p.o.clone()

    (t0, o0), (t1, o1) = timed(-1e30), timed(float("-inf"))
    assert torch.isfinite(o0).all() and torch.equal(o0, o1)
    print(f"  {t0 / 20 * 1e3:.1f} us, {t1 / 20 * 1e3:.1f} us", flush=True)
    assert t1 < 1.5 * t0  # (three passes are done where one does not do)
