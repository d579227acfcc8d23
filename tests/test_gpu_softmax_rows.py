"""Softmax attention of few rows over keys of every kernel's head sizes, as they lie in memory (needs the GPU)."""
import pytest

from paper_2407_10730_amd import seqmix as M
from test_gpu_softmax import Soft, _gpu  # noqa: F401

pytestmark = pytest.mark.gpu


def _behind(p, value):
    """`value` in the rows of k and v behind the sequences' ends (packed: behind the last)."""
    for t in (p.k, p.v):
        if p.page:
            for i, (_, pages) in enumerate(p.where):
                if p.keys[i] % p.page:
                    t[int(pages[-1]), p.keys[i] % p.page:] = value
        else:
            row = t.stride(0)
            t.as_strided((row,), (1,), t.storage_offset() + t.shape[0] * row).fill_(value)


@pytest.mark.parametrize("page", (0, 16, 64))
@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("dv", (64, 128, 256))
@pytest.mark.parametrize("dk", (64, 128, 256))
def test_few_rows_of_every_head_size(dk, dv, dtype, page):
    """Rows in whole 16 bytes of each pair of the kernels' sizes, packed and in pages below and above a tile, many keys in parts
    and few whole; the keys end inside a tile, and nothing behind them counts."""
    for keys in ([301, 45], [2777, 1203], [30, 3]):
        p = Soft([1, 3], keys=keys, heads=4, kv_heads=2, dk=dk, dv=dv, dtype=dtype, page=page, mask="causal")
        assert p.op.plan().kernel == M.SEQMIX_KERNEL_STEP
        assert not page or (p.k.data_ptr() | p.v.data_ptr()) % 16 == 0
        _behind(p, float("nan"))
        p.run().check()
