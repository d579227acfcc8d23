"""Timed cases of the token-mixing operators: linear attention with decay, the causal convolution
over tokens, and the norms around a block fused with its gate and residual scale.

A case is one call of one operator.  `prepare` makes what a program holds before the call (inputs
and states on the GPU, the descriptor, the output tensors), `run` is one call, in plain torch
(`own` false) or through the library (`own` true), `exact` is the definition in float64.
"""
import math

import torch

own = False

_DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _attn(name, lens, heads, qk_heads, dk, dv, dtype, decay, carry):
    """lens: "64x1" (64 sequences of one token) or "100,1,0" (packed sequences of these lengths);
    decay: "token" or "head"; carry: the states come from a pool, by slot, and are updated in place."""
    return {"op": "attn", "lens": lens, "heads": heads, "qk_heads": qk_heads, "dk": dk, "dv": dv,
            "dtype": dtype, "decay": decay, "carry": carry, **({"name": name} if name else {})}


def _conv(name, lens, channels, extra, width, dtype, silu, carry):
    """extra: further columns of the projection that x is a part of; carry: as for attention."""
    return {"op": "conv", "lens": lens, "channels": channels, "extra": extra, "width": width,
            "dtype": dtype, "silu": silu, "carry": carry, **({"name": name} if name else {})}


def _norm(name, rows, width, group, dtype, kind, gate, residual, pre):
    """kind: "rms" or "layer"; gate: "none", "silu" (a value for each element) or "sequence" (a
    sigmoid gate for each channel and run of rows); residual: adds the scaled block to the residual
    stream; pre: norms the sum for the next block too."""
    return {"op": "norm", "rows": rows, "width": width, "group": group, "dtype": dtype, "kind": kind,
            "gate": gate, "residual": residual, "pre": pre, **({"name": name} if name else {})}


def listed():
    return [
        # one decoding step of a few requests: launch latency and 8 MB of states
        _attn("attn_step_few", "8x1", 16, 16, 128, 128, "bf16", "token", True),
        # one decoding step of a full batch: bound by reading and writing the states
        _attn("attn_step_batch", "256x1", 16, 8, 128, 128, "bf16", "token", True),
        # one prompt of ordinary length, decay from the data
        _attn("attn_prompt", "8192", 16, 8, 128, 128, "bf16", "token", False),
        # packed prompts of ragged lengths that continue from carried states, an empty one and one of a
        # single token among them; narrow keys
        _attn("attn_ragged", "1000,1,0,517,2048,63,64,65,129,1777", 12, 4, 64, 128, "bf16", "token", True),
        # one long document, the decay a constant of each head
        _attn("attn_long", "65536", 8, 8, 128, 128, "bf16", "head", False),
        # fp32 with head sizes that fill no tile
        _attn("attn_odd_f32", "777,1300,31", 6, 3, 80, 112, "f32", "token", True),
        # the window of a decoding step
        _conv("conv_step", "64x1", 4096, 2048, 4, "bf16", True, True),
        # q, k and v of a prompt out of the projection
        _conv("conv_prompt", "8192", 4096, 2048, 4, "bf16", True, False),
        # fp32, ragged, odd sizes
        _conv("conv_ragged_f32", "333,1,0,2,900,61", 1001, 0, 3, "f32", False, True),
        # norm of each head of attention's output with its gate
        _norm("norm_heads_gate", 8192, 2048, 128, "bf16", "rms", "silu", False, False),
        # norm after a block, gate and scale, residual sum and the next block's norm
        _norm("norm_residual", 8192, 2048, 2048, "bf16", "rms", "sequence", True, True),
        # the same at one decoding step, fp32 and an odd width
        _norm("norm_step_f32", 13, 1537, 1537, "f32", "layer", "silu", True, True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _odd(rng, lo, hi):
    return _log_int(rng, lo, hi) | 1


def draw(rng):
    while True:
        case = _draw(rng)
        w = work(case)
        if w["bytes"] < 5e8 and w["flops"] < 3e10:  # below the largest listed cases
            return case


def _draw(rng):
    op = rng.choice(("attn", "attn", "conv", "norm"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    form = rng.choice(("step", "prompt", "ragged"))
    if form == "step":
        lens = "%dx1" % _log_int(rng, 1, 256)
    elif form == "prompt":
        lens = str(_odd(rng, 2, 65536 if op == "attn" else 8192))
    else:
        lens = ",".join(str(rng.choice((0, 1, _log_int(rng, 2, 2048), _log_int(rng, 2, 2048))))
                        for _ in range(rng.randint(2, 12)))
        if not any(_lens(lens)):
            lens = "1," + lens
    carry = form != "prompt" or rng.random() < 0.3
    if op == "attn":
        qk = _log_int(rng, 1, 16)
        return _attn(None, lens, qk * rng.choice((1, 1, 2, 4)), qk,
                     rng.choice((32, 64, 64, 80, 96, 128, 128, 192, 256, rng.randint(16, 256))),
                     rng.choice((64, 64, 112, 128, 128, 128, 256, rng.randint(16, 256))),
                     dtype, rng.choice(("token", "token", "head")), carry)
    if op == "conv":
        channels = rng.choice((8 * _odd(rng, 16, 1023), _odd(rng, 64, 8192)))
        return _conv(None, lens, channels, rng.choice((0, 0, 8 * rng.randint(1, 256))), rng.choice((2, 3, 4, 4, 4)),
                     dtype, rng.random() < 0.7, carry)
    rows, kind = _odd(rng, 1, 16384), rng.choice(("rms", "rms", "layer"))
    if rng.random() < 0.4:
        group = rng.choice((64, 128, 128, 256, _odd(rng, 16, 512)))
        return _norm(None, rows, group * rng.choice((1, 2, 4, 5, 8, 16, 20, 32)), group, dtype, kind, "silu", False, False)
    width = rng.choice((8 * _odd(rng, 32, 1023), _odd(rng, 200, 8192)))
    return _norm(None, rows, width, width, dtype, kind, rng.choice(("none", "silu", "sequence")), True,
                 rng.random() < 0.7)


def _lens(text):
    if "x" in text:
        n, t = text.split("x")
        return [int(t)] * int(n)
    return [int(t) for t in text.split(",")]


def work(case):
    es = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "norm":
        n = case["rows"] * case["width"]
        moved = 2 + (case["gate"] == "silu") + case["residual"] + case["pre"]
        return {"bytes": n * es * moved, "flops": 8 * n}
    lens = _lens(case["lens"])
    tokens = sum(lens)
    if case["op"] == "conv":
        window = (2 if case["carry"] else 1) * len(lens) * (case["width"] - 1) * case["channels"]
        return {"bytes": (2 * tokens * case["channels"] + window + case["channels"] * case["width"]) * es,
                "flops": 2 * case["width"] * tokens * case["channels"]}
    h, hq, dk, dv = case["heads"], case["qk_heads"], case["dk"], case["dv"]
    state = len(lens) * h * dk * dv * 4
    return {"bytes": tokens * (2 * hq * dk + 2 * h * dv) * es + tokens * h * 4 * (case["decay"] == "token")
            + state * (2 if case["carry"] else 1),
            "flops": 4 * tokens * h * dk * dv}


def _randn(gen, *shape, scale=1.0):
    return torch.randn(*shape, device="cuda", generator=gen) * scale


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return {"attn": _prepare_attn, "conv": _prepare_conv, "norm": _prepare_norm}[case["op"]](case, gen)


def _packing(case, gen):
    """Where the sequences lie in the packed rows, and the slots of their states in the pool."""
    lens = _lens(case["lens"])
    offsets = torch.tensor([0] + lens, device="cuda").cumsum(0)
    uniform = len(set(lens)) == 1
    slots = len(lens) + 3 if case["carry"] else len(lens)
    index = torch.randperm(slots, device="cuda", generator=gen)[:len(lens)] if case["carry"] else None
    return {"case": case, "lens": lens, "tokens": sum(lens), "offsets": offsets, "slots": slots, "index": index,
            "offsets_arg": None if uniform else offsets,
            "index_arg": None if index is None else index.to(torch.int32)}


def _prepare_attn(case, gen):
    s = _packing(case, gen)
    h, hq, dk, dv, n, dt = case["heads"], case["qk_heads"], case["dk"], case["dv"], s["tokens"], _DT[case["dtype"]]
    # q, k and v are columns of one tensor, as the convolution leaves them; k of unit length
    qkv = torch.empty(n, 2 * hq * dk + h * dv, device="cuda", dtype=dt)
    s["q"], s["k"], s["v"] = (t.view(n, -1, d) for t, d in zip(qkv.split([hq * dk, hq * dk, h * dv], 1), (dk, dk, dv)))
    s["q"].copy_(_randn(gen, n, hq, dk))
    k = _randn(gen, n, hq, dk)
    s["k"].copy_(k / k.square().sum(-1, keepdim=True).sqrt())
    s["v"].copy_(_randn(gen, n, h, dv))
    if case["decay"] == "token":  # log of a sigmoid, most of them near zero: memories of some to some hundred tokens
        s["decay"] = torch.nn.functional.logsigmoid(_randn(gen, n, h) + 2) / 8
    else:  # 1 - 2^-5, 1 - 2^-6, ...
        s["decay"] = torch.log1p(-torch.exp2(-5 - torch.arange(h, device="cuda") % 8 * 1.0)) * (0.9 + 0.2 * torch.rand(
            h, device="cuda", generator=gen))
    s["state"] = _randn(gen, s["slots"], h, dk, dv, scale=0.3) if case["carry"] else None
    s["out_state"] = s["state"] if case["carry"] else torch.empty(s["slots"], h, dk, dv, device="cuda")
    s["o"] = torch.empty(n, h, dv, device="cuda", dtype=dt)
    s["scale"] = dk ** -0.5
    if own:
        from paper_2407_10730_amd import seqmix
        s["handle"] = seqmix.LinearAttention(
            tokens=n, seqs=len(s["lens"]), slots=s["slots"], heads=h, qk_heads=hq, dk=dk, dv=dv, dtype=case["dtype"],
            decay=case["decay"], scale=s["scale"], q_strides=s["q"].stride()[:2], k_strides=s["k"].stride()[:2],
            v_strides=s["v"].stride()[:2])
    return s


def _prepare_conv(case, gen):
    s = _packing(case, gen)
    c, w, n, dt = case["channels"], case["width"], s["tokens"], _DT[case["dtype"]]
    s["x"] = _randn(gen, n, c + case["extra"]).to(dt)[:, :c]
    s["w"] = _randn(gen, c, w, scale=w ** -0.5).to(dt)
    s["bias"] = _randn(gen, c, scale=0.1)
    s["window"] = _randn(gen, s["slots"], w - 1, c).to(dt) if case["carry"] else None
    s["out_window"] = s["window"] if case["carry"] else torch.empty(s["slots"], w - 1, c, device="cuda", dtype=dt)
    s["y"] = torch.empty(n, c, device="cuda", dtype=dt)
    # rows of [windows; x] that each token's taps read, and that the new windows hold (plain form); -1: none
    row, first = torch.arange(n, device="cuda"), s["offsets"][:-1].repeat_interleave(
        torch.tensor(s["lens"], device="cuda"))
    seq = torch.arange(len(s["lens"]), device="cuda").repeat_interleave(torch.tensor(s["lens"], device="cuda"))
    tap = torch.arange(w, device="cuda") - (w - 1)
    s["taps"] = _tap_rows(row[:, None] - first[:, None] + tap, first[:, None], seq[:, None], w, s)
    last = (s["offsets"][1:] - s["offsets"][:-1])[:, None] + tap[:-1] + 1
    seq = torch.arange(len(s["lens"]), device="cuda")[:, None]
    s["tail"] = _tap_rows(last - 1, s["offsets"][:-1, None], seq, w, s)
    if own:
        from paper_2407_10730_amd import seqmix
        s["handle"] = seqmix.TokenConv(tokens=n, seqs=len(s["lens"]), slots=s["slots"], channels=c, width=w,
                                       dtype=case["dtype"], act="silu" if case["silu"] else "none", bias=True,
                                       x_row=s["x"].stride(0))
    return s


def _tap_rows(t, first, seq, w, s):
    """Row of [windows; x] of token t (before a sequence's start: in its window) of each sequence."""
    at = s["slots"] * (w - 1) + first + t
    if s["case"]["carry"]:
        return torch.where(t >= 0, at, s["index"][seq] * (w - 1) + (w - 1) + t)
    return torch.where(t >= 0, at, -1)


def _prepare_norm(case, gen):
    n, d, g, dt = case["rows"], case["width"], case["group"], _DT[case["dtype"]]
    s = {"case": case, "eps": 1e-6}
    s["u"] = (_randn(gen, n, d) * torch.exp(_randn(gen, n, 1))).to(dt)
    s["w"], s["b"] = 1 + _randn(gen, g, scale=0.2), _randn(gen, g, scale=0.2) if case["kind"] == "layer" else None
    s["run"] = 1
    s["gate"] = None
    if case["gate"] == "silu":
        s["gate"] = _randn(gen, n, d).to(dt)
    elif case["gate"] == "sequence":
        s["run"] = 512
        s["gate"] = _randn(gen, -(-n // 512), d).to(dt)
    s["res"] = _randn(gen, n, d, scale=3.0).to(dt) if case["residual"] else None
    s["scale"] = 0.7
    s["scale_vec"] = 0.1 + torch.rand(d, device="cuda", generator=gen) if case["residual"] else None
    s["pw"] = 1 + _randn(gen, d, scale=0.2) if case["pre"] else None
    s["pb"] = _randn(gen, d, scale=0.2) if case["pre"] and case["kind"] == "layer" else None
    s["y"] = torch.empty(n, d, device="cuda", dtype=dt)
    s["h"] = torch.empty(n, d, device="cuda", dtype=dt) if case["pre"] else None
    if own:
        from paper_2407_10730_amd import seqmix
        act = {"none": "none", "silu": "silu", "sequence": "sigmoid"}[case["gate"]]
        s["handle"] = seqmix.GateNorm(rows=n, width=d, group=g, dtype=case["dtype"], post=case["kind"],
                                      post_bias=s["b"] is not None, gate=act, gate_run=s["run"],
                                      residual=case["residual"], scale=s["scale"],
                                      scale_vec=s["scale_vec"] is not None, pre=case["kind"] if case["pre"] else "none",
                                      pre_bias=s["pb"] is not None, eps=s["eps"])
    return s


def run(s):
    op = s["case"]["op"]
    if op == "attn":
        if own:
            s["handle"].run(s["q"], s["k"], s["v"], s["decay"], s["state"], s["out_state"], s["o"],
                            offsets=s["offsets_arg"], slot_index=s["index_arg"])
            return {"o": s["o"], "state": s["out_state"]}
        return _plain_attn(s)
    if op == "conv":
        if own:
            s["handle"].run(s["x"], s["w"], s["bias"], s["window"], s["out_window"], s["y"],
                            offsets=s["offsets_arg"], slot_index=s["index_arg"])
            return {"y": s["y"], "window": s["out_window"]}
        return _plain_conv(s)
    if own:
        s["handle"].run(s["u"], s["w"], s["b"], s["gate"], s["res"], s["scale_vec"], s["pw"], s["pb"], s["y"], s["h"])
        return {"y": s["y"], "h": s["h"]} if s["h"] is not None else {"y": s["y"]}
    return _plain_norm(s)


def _range_sums(g):
    """[..., i, j] = g_{j+1} + ... + g_i for i >= j, -inf above the diagonal."""
    n = g.shape[-1]
    lower = torch.ones(n, n, dtype=torch.bool, device=g.device).tril()
    below = torch.where(lower.tril(-1), g[..., :, None], 0.0).cumsum(-2)
    return torch.where(lower, below, -math.inf)


def _plain_attn(s):
    """Chunks of 64 tokens: scores within a chunk, and a matrix of decays from chunk to chunk."""
    case, lens = s["case"], s["lens"]
    h, hq, dk, dv = case["heads"], case["qk_heads"], case["dk"], case["dv"]
    longest = max(lens)
    size = 64 if longest > 64 else longest
    chunks = -(-longest // size)
    at = torch.arange(chunks * size, device="cuda")
    live = at < (s["offsets"][1:] - s["offsets"][:-1])[:, None]
    rows = torch.where(live, s["offsets"][:-1, None] + at, 0)

    def chunked(x, n):  # [tokens, heads, n] -> [seqs, heads, chunks, size, n] in 32 bits, zeros past the ends
        x = torch.where(live[..., None, None], x[rows].float(), 0.0)
        x = x.repeat_interleave(h // x.shape[2], 2).transpose(1, 2)
        return x.reshape(len(lens), h, chunks, size, n)

    q, k, v = chunked(s["q"], dk), chunked(s["k"], dk), chunked(s["v"], dv)
    g = s["decay"][:, :, None] if case["decay"] == "token" else s["decay"][None, :, None].expand(s["tokens"], h, 1)
    g = chunked(g, 1)[..., 0]
    decays = _range_sums(g)
    scores = torch.matmul(q, k.transpose(-1, -2).contiguous()) * decays.exp()
    o = torch.matmul(scores, v)
    added = torch.matmul((k * decays[..., -1, :, None].exp()).transpose(-1, -2).contiguous(), v)
    first = s["state"][s["index"]] if case["carry"] else torch.zeros(len(lens), h, dk, dv, device="cuda")
    added = torch.cat([first[:, :, None], added], 2).flatten(3)
    across = torch.nn.functional.pad(g.sum(-1), (1, 0))
    states = torch.matmul(_range_sums(across).exp(), added).reshape(len(lens), h, chunks + 1, dk, dv)
    o = o + g.cumsum(-1).exp()[..., None] * torch.matmul(q, states[:, :, :-1])
    o = (o * s["scale"]).reshape(len(lens), h, chunks * size, dv).transpose(1, 2)
    s["o"].copy_(o[live])
    if case["carry"]:
        s["out_state"][s["index"]] = states[:, :, -1]
    else:
        s["out_state"].copy_(states[:, :, -1])
    return {"o": s["o"], "state": s["out_state"]}


def _plain_conv(s):
    case = s["case"]
    c, w = case["channels"], case["width"]
    window = s["window"] if case["carry"] else torch.zeros_like(s["out_window"])
    rows = torch.cat([window.reshape(-1, c), s["x"], s["x"].new_zeros(1, c)])
    y = s["bias"] + (rows[s["taps"]].float() * s["w"].float().t()).sum(1)
    if case["silu"]:
        y = y / (1 + (-y).exp())
    new = rows[s["tail"]]
    s["y"].copy_(y)
    if case["carry"]:
        s["out_window"][s["index"]] = new
    else:
        s["out_window"].copy_(new)
    return {"y": s["y"], "window": s["out_window"]}


def _plain_norm(s):
    case = s["case"]
    n, d, g = case["rows"], case["width"], case["group"]

    def norm(x, w, b):
        if case["kind"] == "layer":
            x = x - x.mean(-1, keepdim=True)
        x = x * (x.square().mean(-1, keepdim=True) + s["eps"]).rsqrt() * w
        return x if b is None else x + b

    y = norm(s["u"].float().view(n, d // g, g), s["w"], s["b"]).view(n, d)
    if s["gate"] is not None:
        gate = s["gate"].float()
        on = 1 / (1 + (-gate).exp())
        on = on * gate if case["gate"] == "silu" else on
        y = y * on.repeat_interleave(s["run"], 0)[:n]
    y = y * s["scale"]
    if case["residual"]:
        y = s["res"].float() + s["scale_vec"] * y
    s["y"].copy_(y)
    if not case["pre"]:
        return {"y": s["y"]}
    s["h"].copy_(norm(y, s["pw"], s["pb"]))
    return {"y": s["y"], "h": s["h"]}


def exact(case, seed):
    s = prepare(case, seed)
    return {"attn": _exact_attn, "conv": _exact_conv, "norm": _exact_norm}[case["op"]](case, s)


def _exact_attn(case, s):
    """The recurrence, token by token; sequences side by side while they last."""
    lens, h, dk, dv = s["lens"], case["heads"], case["dk"], case["dv"]
    elements = len(lens) * h * dk * dv
    if max(lens) * (3e-5 + elements * 8 * 8 / 3e12) > 15:
        return None
    q, k, v = s["q"].double(), s["k"].double(), s["v"].double()
    rep = h // case["qk_heads"]
    state = s["state"][s["index"]].double() if case["carry"] else torch.zeros(len(lens), h, dk, dv, device="cuda",
                                                                            dtype=torch.float64)
    order = sorted(range(len(lens)), key=lambda i: -lens[i])  # the longest first: those that go on are a prefix
    state = state[order]
    start = [int(x) for x in s["offsets"][:-1].tolist()]
    starts = torch.tensor([start[i] for i in order], device="cuda")
    o = torch.zeros(s["tokens"], h, dv, device="cuda", dtype=torch.float64)
    fade = s["decay"].double().exp()
    for t in range(max(lens)):
        m = sum(lens[i] > t for i in order)
        rows = starts[:m] + t
        part = state[:m]
        part.mul_(fade[rows][..., None, None] if case["decay"] == "token" else fade[:, None, None])
        kt = k[rows].repeat_interleave(rep, 1) if rep > 1 else k[rows]
        part.addcmul_(kt[..., None], v[rows][..., None, :])
        qt = q[rows].repeat_interleave(rep, 1) if rep > 1 else q[rows]
        o[rows] = (qt[..., None] * part).sum(-2)
    back = torch.empty_like(state)
    back[order] = state
    if not case["carry"]:
        return {"o": o * s["scale"], "state": back}
    pool = s["state"].double()
    pool[s["index"]] = back
    return {"o": o * s["scale"], "state": pool}


def _exact_conv(case, s):
    c, w = case["channels"], case["width"]
    x, weight, bias = s["x"].double(), s["w"].double(), s["bias"].double()
    pool = s["window"].double() if case["carry"] else torch.zeros(s["slots"], w - 1, c, device="cuda",
                                                                  dtype=torch.float64)
    y, first = [], 0
    for i, n in enumerate(s["lens"]):
        slot = int(s["index"][i]) if case["carry"] else i
        rows = torch.cat([pool[slot], x[first:first + n]])
        z = bias.expand(n, c).clone()
        for j in range(w):
            z += weight[:, j] * rows[j:j + n]
        y.append(z * torch.sigmoid(z) if case["silu"] else z)
        pool[slot] = rows[n:]
        first += n
    return {"y": torch.cat(y), "window": pool}


def _exact_norm(case, s):
    n, d, g, eps = case["rows"], case["width"], case["group"], s["eps"]

    def norm(x, w, b):
        mean = x.sum(-1, keepdim=True) / x.shape[-1] if case["kind"] == "layer" else 0.0
        var = ((x - mean) ** 2).sum(-1, keepdim=True) / x.shape[-1]
        y = (x - mean) / torch.sqrt(var + eps) * w.double()
        return y + b.double() if b is not None else y

    y = norm(s["u"].double().reshape(n * (d // g), g), s["w"], s["b"]).reshape(n, d)
    if s["gate"] is not None:
        z = s["gate"].double()[torch.arange(n, device="cuda") // s["run"]]
        y = y * torch.sigmoid(z) * (z if case["gate"] == "silu" else 1.0)
    y = y * s["scale"]
    if case["residual"]:
        y = s["res"].double() + s["scale_vec"].double() * y
    return {"y": y, "h": norm(y, s["pw"], s["pb"])} if case["pre"] else {"y": y}
