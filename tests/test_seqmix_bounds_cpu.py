"""The bound of attention's outputs tells a wrong sum from a rounding: mistakes planted in the definition pass it."""
import numpy as np
import pytest

from oracle import seqmix as ref


def _bf16(x):
    b = x.astype(np.float32).view(np.uint32)
    return ((b + 0x7fff + ((b >> 16) & 1)) & np.uint32(0xffff0000)).view(np.float32).astype(np.float64)


def _problem(tokens, decay, dk=64, dv=64):
    rng = np.random.default_rng(tokens)
    q, v = (_bf16(rng.standard_normal((tokens, 1, d))) for d in (dk, dv))
    k = _bf16(rng.standard_normal((tokens, 1, dk)) * dk ** -0.5)
    g = -np.exp(rng.standard_normal((tokens, 1)) * 1.5 - 3) if decay else np.zeros((tokens, 1))
    return q, k, v, g, rng.standard_normal((1, 1, dk, dv))


def _scores(q, k, g):
    """Of a chunk that is all the tokens, below the diagonal."""
    b = np.cumsum(g[:, 0])
    return np.tril((q[:, 0] @ k[:, 0].T) * np.exp(np.minimum(b[:, None] - b[None], 0.0)))


@pytest.mark.parametrize("tokens", [33, 64])
@pytest.mark.parametrize("decay", [False, True])
@pytest.mark.parametrize("mistake", [None, "tile", "scores", "state rounded", "scores rounded"])
def test_bound_tells_mistakes(tokens, decay, mistake):
    q, k, v, g, state = _problem(tokens, decay)
    o, o_abs, _, _ = ref.linear_attention(q, k, v, g, [tokens], state, 1.0)
    p, first = _scores(q, k, g), state[0, 0]
    if mistake == "tile":
        p[tokens - tokens % 16 - 16:, :16] = 0.0
    elif mistake == "scores":
        p *= 0.95
    elif mistake == "scores rounded":
        p = _bf16(p)
    elif mistake == "state rounded":
        first = _bf16(first)
    got = np.exp(np.cumsum(g[:, 0]))[:, None] * (q[:, 0] @ first) + p @ v[:, 0]
    exact = np.abs(got - o[:, 0]) <= ref.attention_bound(o, o_abs, tokens, 64, "bf16", "f32", True)[:, 0]
    assert exact.all() == (mistake is None)
    rounded = np.abs(_bf16(got) - o[:, 0]) <= ref.attention_bound(o, o_abs, tokens, 64, "bf16", "bf16", True)[:, 0]
    assert rounded.all() == (mistake is None)
