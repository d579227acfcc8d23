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


def sees(mask, n, keys, tree=None):
    """[n, keys]: which keys each of a sequence's n rows sees.  tree: the rows' masks as Python numbers of 64 bits."""
    own = np.arange(keys) - (keys - n)
    if mask == "full":
        return np.ones((n, keys), bool)
    if mask == "causal":
        return own[None] <= np.arange(n)[:, None]
    bits = [[i < 0 or (i < 64 and (int(m) >> int(i)) & 1 == 1) for i in own] for m in tree]
    return np.array(bits, bool).reshape(n, keys)


def softmax_attention(q, k, v, on, scale):
    """One sequence.  q: [n, H, dk], k: [m, Hk, dk], v: [m, Hk, dv], on: [n, m].  Returns o, the same sums over |v|, and for each row
    and head the largest |scale| sum |q| |k| of the keys that it sees."""
    n, heads = q.shape[:2]
    rep = heads // k.shape[1]
    o, o_abs, most = np.zeros((n, heads, v.shape[2])), np.zeros((n, heads, v.shape[2])), np.zeros((n, heads))
    for t in range(n):
        at = np.nonzero(on[t])[0]
        if not at.size:
            continue
        for h in range(heads):
            kk, vv = k[at, h // rep], v[at, h // rep]
            with np.errstate(all="ignore"):
                s = scale * (kk @ q[t, h])
                p = np.exp(s - s.max())
                p /= p.sum()
                o[t, h] = p @ vv
                o_abs[t, h] = p @ np.abs(vv)
                most[t, h] = abs(scale) * (np.abs(kk) @ np.abs(q[t, h])).max()
    return o, o_abs, most


def softmax_bound(o, o_abs, most, keys, dk, dtype, parts=1):
    """How far outputs may be off, point by point, with u = 2^-24 and r = 2^-8 (half a unit in the last of bf16's 8 bits).

    A score is a sum of dk products, multiplied by the scale (times log2 e, rounded) and lessened by the maximum: off by (dk + 6) u of its
    sum over absolute values, `most` at most; the exponential of it is off by as much, relatively, and 4 u of its own.  The
    weights, and their products with v, are summed over `keys` keys, and rescaled when the maximum moves, by two
    roundings and an exponential (6 u) at most once for 16 keys: (2 keys + 32) u.  The quotient has this error twice.  Weights
    enter products in bf16 as `parts` parts, each the rounding of what the ones before left: r^parts is left out.  A bf16
    output is rounded once: r |o|."""
    u, r = 2.0 ** -24, 2.0 ** -8
    part = 2 * ((dk + 6) * u * most[..., None] + (2 * keys + 32) * u)
    if dtype == "bf16":
        return (part + r ** parts) * (1 + r) * o_abs + r * np.abs(o) + 1e-37
    return part * o_abs + 1e-37


def rotary(x, position, freqs, rot, layout, amplitude):
    """x: [T, H, d], position: [T], freqs: [rot / 2]."""
    y = x.copy()
    w = np.outer(position.astype(np.float64), freqs)[:, None]
    a = x[..., :rot // 2] if layout == "half" else x[..., 0:rot:2]
    b = x[..., rot // 2:rot] if layout == "half" else x[..., 1:rot:2]
    at = (slice(0, rot // 2), slice(rot // 2, rot)) if layout == "half" else (slice(0, rot, 2), slice(1, rot, 2))
    y[..., at[0]] = amplitude * (a * np.cos(w) - b * np.sin(w))
    y[..., at[1]] = amplitude * (b * np.cos(w) + a * np.sin(w))
    return y


class Pages:
    """The pages of a cache's requests, one token at a time."""

    def __init__(self, lens, table, free_pages, taken, page):
        self.lens, self.table, self.free, self.taken, self.page = list(lens), [list(r) for r in table], list(free_pages), taken, page

    def pages(self, n):
        return -(-n // self.page)

    def move(self, slots, kept, new):
        """slots: of each sequence (None: skipped); kept: None or what each goes back to; new: rows that each gets.
        Returns place, position (of all new rows) and admitted."""
        gone = []
        for i, s in enumerate(slots):
            if s is None:
                continue
            keep = self.lens[s] if kept is None else max(0, min(kept[i], self.lens[s]))
            gone += self.table[s][self.pages(keep):self.pages(self.lens[s])]
            self.lens[s] = keep
        self.taken -= len(gone)
        self.free[self.taken:self.taken + len(gone)] = gone
        place, position, admitted, full = [], [], [], False
        for s, n in zip(slots, new):
            want = 0 if s is None else self.pages(self.lens[s] + n) - self.pages(self.lens[s])
            room = s is not None and self.pages(self.lens[s] + n) <= len(self.table[s])
            full |= room and want > 0 and self.taken + want > len(self.free)
            if not room or (want and full):
                place += [-1] * n
                position += [0] * n
                admitted.append(-1)
                continue
            first = self.pages(self.lens[s])
            self.table[s][first:first + want] = self.free[self.taken:self.taken + want]
            self.taken += want
            for t in range(self.lens[s], self.lens[s] + n):
                place.append(self.table[s][t // self.page] * self.page + t % self.page)
                position.append(t)
            self.lens[s] += n
            admitted.append(s)
        return place, position, admitted
