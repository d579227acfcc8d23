"""Sizes that softmax attention refuses, and the largest that it takes."""
import pytest

from paper_2407_10730_amd import binding as B
from paper_2407_10730_amd import seqmix as M

MOST = (1 << 31) - 1024


def _create(**kw):
    base = dict(tokens=2, seqs=2, slots=2, heads=1, dk=8, key_tokens=2)
    base.update(kw)
    return M.SoftmaxAttention(**base)


@pytest.mark.parametrize("kw", [
    dict(key_tokens=MOST), dict(page=1, pages=1, max_pages=MOST), dict(page=64, pages=8, max_pages=MOST // 64),
    dict(tokens=MOST - 2), dict(tokens=MOST // 3 - 2, heads=3),
])
def test_keys_are_numbered_in_32_bits(kw):
    """Loops over keys step past the last by less than 1024: the largest sizes are taken, one more is refused (they would count past
    2^31 and not end)."""
    _create(**kw)
    name = next(n for n in ("key_tokens", "max_pages", "tokens") if n in kw)
    with pytest.raises(B.Conv2dError) as e:
        _create(**{**kw, name: kw[name] + 1})
    assert e.value.status == B.CONV2D_E_UNSUPPORTED


@pytest.mark.parametrize("scale", (2.4e38, -3.4e38))
def test_scales_that_are_infinite_as_powers_of_two(scale):
    """Scores are multiplied by scale log2(e): a finite scale above 2^128 / log2(e) made a score of zero NaN."""
    _create(scale=2.3e38 if scale > 0 else -2.3e38)
    with pytest.raises(B.Conv2dError) as e:
        _create(scale=scale)
    assert e.value.status == B.CONV2D_E_INVALID
