"""Layers on the library's operators: prompts, prompts that continue, single tokens.

Gated linear attention:
    h      = rmsnorm(x)
    q k v z g = project(h)                       1x1 convolution (conv2d, channels last)
    q k v  = silu(causal convolution(q k v))     window carried per request
    o      = linear attention(q, k, v, decay g)  state carried per request
    u      = project(rmsnorm per head(o) * silu(z))
    x'     = x + scale * rmsnorm(u)              and the next layer's h in the same kernel

Softmax attention over a cache in pages, also of drafted tokens:

    h      = rmsnorm(x)
    q k v  = project(h)                          1x1 convolution
    q k    = rotary positions(q k)               k and v into the cache's pages, given out per request
    o      = softmax attention(q, pages)
    u      = project(o)
    x'     = x + scale * rmsnorm(u)              and the next layer's h in the same kernel

``python -m paper_2407_10730_amd.mixer`` runs packed prompts through one of each, then single tokens of all
requests, and prints the time of each.
"""
from __future__ import annotations

import argparse
from collections import OrderedDict

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

    def close(self):
        if self.desc:
            desc, self.desc = self.desc, 0
            B.conv2d_desc_destroy(desc)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class _Plan:
    """A call size's descriptors, and by stream the tensors between its operators."""

    def __init__(self, **ops):
        self.ops, self.between, self.captured = ops, {}, False


class _Layer:
    """What layers share: the descriptors of the `plans` sizes of calls that were used last, and of those that a graph was
    captured of; by stream a place for what lies between the operators."""

    def __init__(self, device, plans):
        import torch
        self.torch, self.device = torch, torch.device(device)
        self.plans, self._plans, self._places = plans, OrderedDict(), {}

    def _operators(self, tokens, seqs, *kind):
        """The descriptors of calls of this size."""
        raise NotImplementedError

    def _plan(self, capturing, *size):
        p = self._plans.get(size)
        if p is None:
            p = self._plans[size] = _Plan(**self._operators(*size))
            if len(self._plans) > self.plans and not capturing:  # (freeing a workspace is no work for a capture)
                old = next((k for k, q in self._plans.items() if not q.captured and q is not p), None)
                if old:
                    for op in self._plans.pop(old).ops.values():
                        op.close()
        self._plans.move_to_end(size)
        p.captured |= capturing
        return p

    def _views(self, *parts):
        """From the tensors [tokens, columns] between the operators what a call uses."""
        return parts

    def _between(self, p, tokens, stream, capturing, columns):
        """The tensors between the operators, on `stream`."""
        t = None if capturing else p.between.get(stream)
        if t is None:
            sizes = [-(-tokens * c // 64) * 64 for c in columns]
            place = None if capturing else self._places.get(stream)
            if place is None or place.numel() < sum(sizes):
                place = self.torch.empty(sum(sizes), device=self.device, dtype=self.torch.bfloat16)
                if not capturing:
                    self._places[stream] = place
                    for q in self._plans.values():  # the former place goes
                        q.between.pop(stream, None)
            t = self._views(*(part[:tokens * c].view(tokens, c) for part, c in zip(place[:sum(sizes)].split(sizes), columns)))
            if not capturing:
                p.between[stream] = t
        return t


class MixerLayer(_Layer):
    """The layer's weights (random), and the windows and states of up to `slots` requests.

    Descriptors are kept for the `plans` sizes of calls that were used last, and for those that a graph was captured of.
    What lies between the operators has a place for each stream, as large as the largest call there, so calls of disjoint
    slots may run on several streams; a captured call has its own.
    """

    def __init__(self, width=1024, heads=8, qk_heads=4, dk=64, dv=128, taps=4, slots=32, scale=0.5, device="cuda:0",
                 seed=0, plans=32):
        super().__init__(device, plans)
        torch = self.torch
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

    def _operators(self, tokens, seqs):
        cols = self.columns
        return dict(
            norm=seqmix.GateNorm(rows=tokens, width=self.width, post="none", pre="rms"),
            w_in=Projection(tokens, self.w_in), w_out=Projection(tokens, self.w_out),
            conv=seqmix.TokenConv(tokens=tokens, seqs=seqs, slots=self.slots, channels=self.mixed, width=self.taps,
                                  x_row=cols),
            attn=seqmix.LinearAttention(
                tokens=tokens, seqs=seqs, slots=self.slots, heads=self.heads, qk_heads=self.qk_heads, dk=self.dk,
                dv=self.dv, scale=self.dk ** -0.5, q_strides=(self.mixed, self.dk), k_strides=(self.mixed, self.dk),
                v_strides=(self.mixed, self.dv)),
            gate=seqmix.GateNorm(rows=tokens, width=self.inner, group=self.dv, gate="silu", gate_row=cols),
            sum=seqmix.GateNorm(rows=tokens, width=self.width, residual=True, scale=self.scale, pre="rms"))

    def _views(self, h, proj, mix, o, g, u):
        tokens, qk = h.shape[0], self.qk_heads * self.dk
        q, k, v = (part.view(tokens, -1, d) for part, d in zip(mix.split([qk, qk, self.inner], 1),
                                                               (self.dk, self.dk, self.dv)))
        mixed, z, logits = proj[:, :self.mixed + self.inner + self.heads].split([self.mixed, self.inner, self.heads], 1)
        return h, proj, mixed, z, logits, mix, q, k, v, o, o.view(tokens, self.heads, self.dv), g, u

    def run(self, x, slot_index, offsets=None):
        """x: [tokens, width] bf16, packed; offsets: int64 [requests + 1] (None: equal lengths, so one token each for
        a decoding step); slot_index: int32 [requests].  Windows and states of those slots move on.
        Returns x' and the next layer's normed input; of a request whose slot is outside the pool (an empty place), x' is x."""
        torch, tokens = self.torch, x.shape[0]
        capturing, stream = torch.cuda.is_current_stream_capturing(), torch.cuda.current_stream(self.device)
        p = self._plan(capturing, tokens, slot_index.numel())
        h, proj, mixed, z, logits, mix, q, k, v, o, o_heads, g, u = self._between(
            p, tokens, stream.cuda_stream, capturing, (self.width, self.columns, self.mixed, self.inner, self.inner, self.width))
        op = p.ops
        op["norm"].run(x, pre_w=self.n_in, h=h)
        op["w_in"].run(h, proj, stream)
        decay = torch.nn.functional.logsigmoid(logits.float() + 2) / 8
        op["conv"].run(mixed, self.w_taps, self.b_taps, self.windows, self.windows, mix, offsets=offsets, slot_index=slot_index)
        o.zero_()  # rows of empty places stay so
        op["attn"].run(q, k, v, decay, self.states, self.states, o_heads, offsets=offsets, slot_index=slot_index)
        op["gate"].run(o, self.n_head, gate=z, y=g)
        op["w_out"].run(g, u, stream)
        y, h = torch.empty_like(x), torch.empty_like(x)
        op["sum"].run(u, self.n_out, residual=x, pre_w=self.n_next, y=y, h=h)
        return y, h

    def clear(self, slot_index):
        """A request starts anew in these slots."""
        self.windows[slot_index.long()] = 0
        self.states[slot_index.long()] = 0


class Pages(_Layer):
    """Which pages of the caches each of up to `slots` requests has: one for all SoftmaxLayers of a model, moved on once per
    call of the model.  Calls are kept in order by the caller (all write the same lists)."""

    def __init__(self, slots=32, page=64, pages=2048, max_pages=512, device="cuda:0", plans=32):
        super().__init__(device, plans)
        self.slots, self.page, self.pages, self.max_pages = slots, page, pages, max_pages
        self.lens, self.table, self.free, self.taken = seqmix.CachePages.empty(slots, pages, max_pages, device=self.device)

    def _operators(self, tokens, seqs):
        return dict(pages=seqmix.CachePages(tokens=tokens, seqs=seqs, slots=self.slots, page=self.page, pages=self.pages,
                                            max_pages=self.max_pages))

    def step(self, tokens, slot_index, offsets=None, kept=None):
        """Room for `tokens` new rows of the requests in slot_index, behind the kept[i] rows (int32 [requests], None: all) that
        each still has: place, position (of each row) and admitted (slot_index, -1 where there is no room left).
        A request ends with no new rows and kept 0."""
        torch, capturing = self.torch, self.torch.cuda.is_current_stream_capturing()
        p = self._plan(capturing, tokens, slot_index.numel())
        place, position = torch.empty(2, tokens, device=self.device, dtype=torch.int32)
        admitted = torch.empty_like(slot_index)
        p.ops["pages"].run(kept, self.lens, self.table, self.free, self.taken, place, position, admitted, offsets=offsets,
                           slot_index=slot_index)
        return place, position, admitted


class SoftmaxLayer(_Layer):
    """The layer's weights (random), and its cache of the pages that `pages` (Pages) gives out.

    Descriptors and places are kept as MixerLayer's are; calls on several streams need events between them, as they share
    the cache and the descriptors' workspaces."""

    def __init__(self, pages, width=1024, heads=8, kv_heads=2, dim=128, scale=0.5, base=10000.0, seed=0, plans=32):
        super().__init__(pages.device, plans)
        torch = self.torch
        self.pages, self.width, self.heads, self.kv_heads, self.dim, self.scale = pages, width, heads, kv_heads, dim, scale
        self.inner = heads * dim
        self.columns = self.inner + 2 * kv_heads * dim
        gen = torch.Generator(device=self.device).manual_seed(seed)

        def randn(*shape, scale=1.0, dtype=torch.bfloat16):
            return (torch.randn(*shape, device=self.device, generator=gen) * scale).to(dtype)

        self.w_in = randn(self.columns, width, scale=width ** -0.5)
        self.w_out = randn(width, self.inner, scale=self.inner ** -0.5)
        self.n_in, self.n_out, self.n_next = (1 + randn(width, scale=0.1, dtype=torch.float32) for _ in range(3))
        self.freqs = seqmix.rotary_frequencies(dim, base, device=self.device)
        self.k_cache, self.v_cache = (torch.zeros(pages.pages, pages.page, kv_heads, dim, device=self.device,
                                                  dtype=torch.bfloat16) for _ in range(2))

    def _operators(self, tokens, seqs, mask):
        heads = dict(heads=self.heads, kv_heads=self.kv_heads, dk=self.dim, page=self.pages.page, pages=self.pages.pages)
        row = self.columns, self.dim
        return dict(
            norm=seqmix.GateNorm(rows=tokens, width=self.width, post="none", pre="rms"),
            w_in=Projection(tokens, self.w_in), w_out=Projection(tokens, self.w_out),
            rotary=seqmix.Rotary(tokens=tokens, q_strides=row, k_strides=row, v_strides=row, q_out_strides=row, **heads),
            attn=seqmix.SoftmaxAttention(tokens=tokens, seqs=seqs, slots=self.pages.slots, mask=mask,
                                         max_pages=self.pages.max_pages, q_strides=row, **heads),
            sum=seqmix.GateNorm(rows=tokens, width=self.width, residual=True, scale=self.scale, pre="rms"))

    def _views(self, h, proj, o, u):
        q, k, v = (part.view(h.shape[0], -1, self.dim) for part in proj.split(
            [self.inner, self.kv_heads * self.dim, self.kv_heads * self.dim], 1))
        return h, proj, q, k, v, o, o.view(h.shape[0], self.heads, self.dim), u

    def run(self, x, places, offsets=None, tree=None):
        """x, offsets: as MixerLayer.run takes them; places: what Pages.step returned for these rows; tree: int64 [tokens], the
        drafted rows of its own request that each row sees (None: those up to itself).
        Returns x' and the next layer's normed input; of a request that was not admitted x' is x."""
        torch, tokens = self.torch, x.shape[0]
        place, position, admitted = places
        capturing, stream = torch.cuda.is_current_stream_capturing(), torch.cuda.current_stream(self.device)
        p = self._plan(capturing, tokens, admitted.numel(), "causal" if tree is None else "tree")
        h, proj, q, k, v, o, o_heads, u = self._between(p, tokens, stream.cuda_stream, capturing,
                                                        (self.width, self.columns, self.inner, self.width))
        op, pages = p.ops, self.pages
        op["norm"].run(x, pre_w=self.n_in, h=h)
        op["w_in"].run(h, proj, stream)
        op["rotary"].run(q, k, v, position, self.freqs, q, None, self.k_cache, self.v_cache, place)
        o.zero_()  # rows that were not admitted stay so
        op["attn"].run(q, self.k_cache, self.v_cache, o_heads, offsets=offsets, slot_index=admitted, lens=pages.lens,
                       table=pages.table, tree=tree)
        op["w_out"].run(o, u, stream)
        y, h = torch.empty_like(x), torch.empty_like(x)
        op["sum"].run(u, self.n_out, residual=x, pre_w=self.n_next, y=y, h=h)
        return y, h


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

    pages = Pages(slots=a.requests, pages=a.requests * (a.prompt // 64 + a.steps // 64 + 2), max_pages=a.prompt // 64 + a.steps // 64 + 2)
    soft = SoftmaxLayer(pages)
    none = torch.zeros_like(slots)
    t = timed(lambda: soft.run(x, pages.step(sum(lens), slots, offsets, none), offsets), 10)
    print(f"softmax attention, {sum(lens)} tokens of {a.requests} prompts: {t:.1f} us")
    t = timed(lambda: soft.run(token, pages.step(a.requests, slots)), a.steps)
    print(f"softmax attention, one token each: {t:.1f} us")


if __name__ == "__main__":
    main()
