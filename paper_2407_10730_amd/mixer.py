"""One gated linear-attention layer on the library's operators: prompts, prompts that continue, single tokens.

    h      = rmsnorm(x)
    q k v z g = project(h)                       1x1 convolution (conv2d, channels last)
    q k v  = silu(causal convolution(q k v))     window carried per request
    o      = linear attention(q, k, v, decay g)  state carried per request
    u      = project(rmsnorm per head(o) * silu(z))
    x'     = x + scale * rmsnorm(u)              and the next layer's h in the same kernel

``python -m paper_2407_10730_amd.mixer`` runs packed prompts through it, then single tokens of all
requests, and prints the time of each.
"""
from __future__ import annotations

import argparse

from . import binding as B
from . import seqmix


class Projection:
    """y[rows, K] = x[rows, C] w[K, C]^T as a 1x1 convolution over `rows` pixels, channels last, bf16."""

    def __init__(self, rows, w):
        self.w = w
        k, c = w.shape
        self.desc = B.conv2d_desc_create(B.conv2d_params(
            n=1, c=c, h=rows, w=1, k=k, r=1, s=1, stride_h=1, stride_w=1, pad_h=0, pad_w=0, dil_h=1, dil_w=1, groups=1,
            layout=B.CONV2D_NHWC, x_dtype=B.CONV2D_BF16, y_dtype=B.CONV2D_BF16, has_bias=0))

    def run(self, x, y, stream):
        B.conv2d_fwd(self.desc, x, self.w, None, y, B.CONV2D_ALGO_AUTO, stream)

    def __del__(self):
        try:
            B.conv2d_desc_destroy(self.desc)
        except Exception:
            pass


class MixerLayer:
    """The layer's weights (random), and the windows and states of up to `slots` requests."""

    def __init__(self, width=1024, heads=8, qk_heads=4, dk=64, dv=128, taps=4, slots=32, scale=0.5, device="cuda:0",
                 seed=0):
        import torch
        self.torch, self.device = torch, torch.device(device)
        self.width, self.heads, self.qk_heads, self.dk, self.dv, self.taps, self.slots = (
            width, heads, qk_heads, dk, dv, taps, slots)
        self.scale = scale
        self.mixed = 2 * qk_heads * dk + heads * dv              # q, k and v
        self.inner = heads * dv
        self.columns = -(-(self.mixed + self.inner + heads) // 8) * 8  # ... z and the decay's logits
        gen = torch.Generator(device=self.device).manual_seed(seed)

        def randn(*shape, scale=1.0, dtype=torch.bfloat16):
            return (torch.randn(*shape, device=self.device, generator=gen) * scale).to(dtype)

        self.w_in = randn(self.columns, width, scale=width ** -0.5)
        self.w_out = randn(width, self.inner, scale=self.inner ** -0.5)
        self.w_taps, self.b_taps = randn(self.mixed, taps, scale=taps ** -0.5), randn(self.mixed, scale=0.1, dtype=torch.float32)
        self.n_in, self.n_head, self.n_out = (1 + randn(n, scale=0.1, dtype=torch.float32) for n in (width, dv, width))
        self.n_next = 1 + randn(width, scale=0.1, dtype=torch.float32)
        self.windows = torch.zeros(slots, taps - 1, self.mixed, device=self.device, dtype=torch.bfloat16)
        self.states = torch.zeros(slots, heads, dk, dv, device=self.device)
        self._plans = {}

    def _plan(self, tokens, seqs):
        """Descriptors and buffers of a call's sizes."""
        plan = self._plans.get((tokens, seqs))
        if plan is None:
            torch, cols, bf16 = self.torch, self.columns, self.torch.bfloat16
            new = lambda n: torch.empty(tokens, n, device=self.device, dtype=bf16)  # noqa: E731
            p = {"h": new(self.width), "p": new(cols), "c": new(self.mixed), "o": new(self.inner), "g": new(self.inner),
                 "u": new(self.width)}
            p["norm"] = seqmix.GateNorm(rows=tokens, width=self.width, post="none", pre="rms")
            p["in"], p["out"] = Projection(tokens, self.w_in), Projection(tokens, self.w_out)
            p["conv"] = seqmix.TokenConv(tokens=tokens, seqs=seqs, slots=self.slots, channels=self.mixed, width=self.taps,
                                         x_row=cols)
            qk = self.qk_heads * self.dk
            p["qkv"] = [t.view(tokens, -1, d) for t, d in zip(p["c"].split([qk, qk, self.inner], 1),
                                                             (self.dk, self.dk, self.dv))]
            p["attn"] = seqmix.LinearAttention(
                tokens=tokens, seqs=seqs, slots=self.slots, heads=self.heads, qk_heads=self.qk_heads, dk=self.dk, dv=self.dv,
                scale=self.dk ** -0.5, **{f"{n}_strides": t.stride()[:2] for n, t in zip("qkv", p["qkv"])})
            p["gate"] = seqmix.GateNorm(rows=tokens, width=self.inner, group=self.dv, gate="silu", gate_row=cols)
            p["sum"] = seqmix.GateNorm(rows=tokens, width=self.width, residual=True, scale=self.scale, pre="rms")
            plan = self._plans[(tokens, seqs)] = p
        return plan

    def run(self, x, slot_index, offsets=None):
        """x: [tokens, width] bf16, packed; offsets: int64 [requests + 1] (None: equal lengths, so one token each for
        a decoding step); slot_index: int32 [requests].  Windows and states of those slots move on.
        Returns x' and the next layer's normed input."""
        torch = self.torch
        p = self._plan(x.shape[0], slot_index.numel())
        stream = torch.cuda.current_stream(self.device)
        p["norm"].run(x, pre_w=self.n_in, h=p["h"])
        p["in"].run(p["h"], p["p"], stream)
        mixed, z, logits = p["p"][:, :self.mixed], p["p"][:, self.mixed:self.mixed + self.inner], p["p"][
            :, self.mixed + self.inner:self.mixed + self.inner + self.heads]
        decay = torch.nn.functional.logsigmoid(logits.float() + 2) / 8
        p["conv"].run(mixed, self.w_taps, self.b_taps, self.windows, self.windows, p["c"], offsets=offsets,
                      slot_index=slot_index)
        q, k, v = p["qkv"]
        p["attn"].run(q, k, v, decay, self.states, self.states, p["o"].view(-1, self.heads, self.dv), offsets=offsets,
                      slot_index=slot_index)
        p["gate"].run(p["o"], self.n_head, gate=z, y=p["g"])
        p["out"].run(p["g"], p["u"], stream)
        y, h = torch.empty_like(x), torch.empty_like(x)
        p["sum"].run(p["u"], self.n_out, residual=x, pre_w=self.n_next, y=y, h=h)
        return y, h

    def clear(self, slot_index):
        """A request starts anew in these slots."""
        self.windows[slot_index.long()] = 0
        self.states[slot_index.long()] = 0


def main(argv=None):
    import torch
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--requests", type=int, default=16)
    ap.add_argument("--prompt", type=int, default=1000, help="longest prompt; the others are shorter")
    ap.add_argument("--steps", type=int, default=64)
    a = ap.parse_args(argv)
    layer = MixerLayer(slots=a.requests)
    lens = [max(1, a.prompt * (i + 1) // a.requests) for i in range(a.requests)]
    offsets = torch.tensor([0] + lens, device="cuda").cumsum(0)
    slots = torch.arange(a.requests, device="cuda", dtype=torch.int32)
    x = torch.randn(sum(lens), layer.width, device="cuda").bfloat16()
    token = torch.randn(a.requests, layer.width, device="cuda").bfloat16()

    def timed(f, n):
        f()
        torch.cuda.synchronize()
        t0, t1 = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        t0.record()
        for _ in range(n):
            f()
        t1.record()
        t1.synchronize()
        return t0.elapsed_time(t1) / n * 1e3

    def prompts():
        layer.clear(slots)
        return layer.run(x, slots, offsets)

    print(f"{sum(lens)} tokens of {a.requests} prompts: {timed(prompts, 10):.1f} us")
    print(f"one token each: {timed(lambda: layer.run(token, slots), a.steps):.1f} us")


if __name__ == "__main__":
    main()
