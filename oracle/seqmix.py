"""float64 definitions of the token-mixing operators (numpy, token by token).

Each returns its outputs and, for each, the same sums over absolute values: rounding errors are
bounded relative to those.
"""
import numpy as np


def linear_attention(q, k, v, g, lens, state, scale):
    """q, k: [T, Hq, dk], v: [T, H, dv], g: [T, H] natural logs of the decay, state: [seqs, H, dk, dv].
    Returns o, its absolute sums, the states left, their absolute sums."""
    heads, rep = v.shape[1], v.shape[1] // k.shape[1]
    o = np.zeros(v.shape)
    o_abs = np.zeros(v.shape)
    left, left_abs = state.astype(np.float64).copy(), np.abs(state.astype(np.float64))
    row = 0
    with np.errstate(invalid="ignore", over="ignore"):
        for i, n in enumerate(lens):
            for t in range(row, row + n):
                for h in range(heads):
                    d = np.exp(g[t, h])
                    kk, qq = k[t, h // rep], q[t, h // rep]
                    left[i, h] = d * left[i, h] + np.outer(kk, v[t, h])
                    left_abs[i, h] = d * left_abs[i, h] + np.outer(np.abs(kk), np.abs(v[t, h]))
                    o[t, h] = scale * (qq @ left[i, h])
                    o_abs[t, h] = abs(scale) * (np.abs(qq) @ left_abs[i, h])
            row += n
    return o, o_abs, left, left_abs


def attention_bound(o, o_abs, tokens, dk, dtype, o_dtype, chunks):
    """How far outputs may be off, point by point, after sequences of up to `tokens` tokens.

    With u = 2^-24 and r = 2^-8 (half a unit in the last of bf16's 8 bits): a term passes through at most two roundings
    per token (decay and sum), one per chunk or key column summed, and an exponential whose argument is rounded:
    (2 tokens + dk + 64) u of the sums over absolute values.  Chunks of bf16 tokens multiply scores and states in bf16
    planes, each holding what the one before left: two planes leave r^2, three (for fp32 outputs) r^3 = u, once for
    the scores and once for the states.  A bf16 output is rounded once: r |o|."""
    u, r = 2.0 ** -24, 2.0 ** -8
    sums = (2 * tokens + dk + 64) * u
    if chunks and dtype == "bf16":
        sums += 2 * (u if o_dtype == "f32" else r * r)
    return sums * o_abs if o_dtype == "f32" else sums * (1 + r) * o_abs + r * np.abs(o)


def silu(x):
    return x / (1.0 + np.exp(-x))


def sigmoid(x):
    return 1.0 / (1.0 + np.exp(-x))


def token_conv(x, w, bias, lens, window, act):
    """x: [T, C], w: [C, W], window: [seqs, W - 1, C].  Returns y, the absolute sums of its
    products, and the windows left."""
    width = w.shape[1]
    y, y_abs = np.zeros(x.shape), np.zeros(x.shape)
    left = window.astype(np.float64).copy()
    row = 0
    for i, n in enumerate(lens):
        rows = np.concatenate([left[i], x[row:row + n]])
        for t in range(n):
            taps = rows[t:t + width]
            y[row + t] = bias + (w.T * taps).sum(0)
            y_abs[row + t] = np.abs(bias) + np.abs(w.T * taps).sum(0)
        left[i] = rows[n:]
        row += n
    return (silu(y) if act == "silu" else y), y_abs, left


def norm(x, kind, w, b, eps):
    """Norm of the last axis, and the size that its rounding errors are relative to."""
    if kind == "none":
        return x, np.abs(x)
    mean = x.mean(-1, keepdims=True) if kind == "layer" else 0.0
    c = x - mean
    r = 1.0 / np.sqrt((c * c).mean(-1, keepdims=True) + eps)
    size = np.abs(x) + (np.abs(x).mean(-1, keepdims=True) if kind == "layer" else 0.0)
    y = c * r * w
    size = size * r * np.abs(w)
    if b is not None:
        y, size = y + b, size + np.abs(b)
    return y, size
