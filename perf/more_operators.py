"""Timed cases of softmax attention and what it is served with: the pages of a cache of keys and values, rotary positions
that are written into it, attention of prompts, and attention of single tokens and drafted trees over the cache.

A case is one call of one operator.  `prepare` makes what a program holds before the call (inputs, cache
and page table on the GPU, the descriptor, the output tensors), `run` is one call, in plain torch (`own` false)
or through the library (`own` true), `exact` is the definition in float64 (whole numbers: counted one by one).
"""
import math

import torch

own = False

_DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _pages(name, requests, before, kept, new, page, short=False):
    """requests: of the batch; before: their longest length so far; kept: how many of the last tokens are taken back at
    most; new: "8x1" style, one length for all, or "500,1,0"; page: tokens of a page; short: the pool has too few."""
    return {"op": "pages", "requests": requests, "before": before, "kept": kept, "new": new, "page": page, "short": short,
            **({"name": name} if name else {})}


def _rotary(name, tokens, heads, kv_heads, dk, dv, rot, layout, dtype, scaled, far, cache):
    """rot: leading elements of a head that turn; scaled: frequencies of a model trained on shorter texts; far: largest
    position; cache: "" (k goes to a tensor) or the page size (k and v go to the cache)."""
    return {"op": "rotary", "tokens": tokens, "heads": heads, "kv_heads": kv_heads, "dk": dk, "dv": dv, "rot": rot,
            "layout": layout, "dtype": dtype, "scaled": scaled, "far": far, "cache": cache, **({"name": name} if name else {})}


def _prompt(name, lens, before, heads, kv_heads, dk, dv, dtype, page):
    """lens: packed prompts; before: the longest run of earlier tokens (0: none), which makes the keys come from the cache, in
    pages of `page` tokens."""
    return {"op": "prompt", "lens": lens, "before": before, "heads": heads, "kv_heads": kv_heads, "dk": dk, "dv": dv,
            "dtype": dtype, "page": page, **({"name": name} if name else {})}


def _step(name, requests, before, ragged, drafts, heads, kv_heads, dk, dv, dtype, page):
    """before: the longest cache, of which requests use different parts where `ragged`; drafts: tokens per request, 1 or a tree
    of so many."""
    return {"op": "step", "requests": requests, "before": before, "ragged": ragged, "drafts": drafts, "heads": heads,
            "kv_heads": kv_heads, "dk": dk, "dv": dv, "dtype": dtype, "page": page, **({"name": name} if name else {})}


def listed():
    return [
        # one decoding step: every request gets a token, some a page; nothing but latency
        _pages("pages_step", 64, 4000, 0, "64x1", 16),
        # a batch whose drafts were partly refused: pages go back and are taken again, 12 tokens each
        _pages("pages_drafts", 200, 3000, 11, "200x12", 16),
        # q and k of one decoding step, k and v into the cache: latency
        _rotary("rotary_step", 64, 16, 4, 128, 128, 128, "half", "bf16", True, 30000, 16),
        # a long prompt with frequencies scaled for long texts, into the cache
        _rotary("rotary_prompt", 8192, 16, 4, 128, 128, 128, "half", "bf16", True, 100000, 64),
        # fp32, neighbouring elements turn, part of the head, sizes that fill no vector, far positions
        _rotary("rotary_odd_f32", 777, 6, 3, 80, 112, 50, "interleaved", "f32", False, 2000000, 0),
        # one long prompt: bound by the matrix cores
        _prompt("prompt_long", "8192", 0, 16, 4, 128, 128, "bf16", 0),
        # packed prompts of ragged lengths, an empty one and single tokens among them, narrow keys
        _prompt("prompt_ragged", "1000,1,0,517,2048,63,64,65,129,1777", 0, 12, 4, 64, 128, "bf16", 0),
        # parts of prompts that go on from what the cache holds
        _prompt("prompt_goes_on", "512,512,300,700", 12000, 16, 4, 128, 128, "bf16", 64),
        # fp32 with head sizes that fill no tile
        _prompt("prompt_odd_f32", "777,1300,31", 0, 6, 3, 80, 112, "f32", 0),
        # one decoding step of a full batch of different lengths: bound by reading the cache
        _step("step_batch", 64, 8000, True, 1, 16, 4, 128, 128, "bf16", 16),
        # one decoding step of two long documents: few rows, a long axis
        _step("step_long", 2, 65536, False, 1, 16, 4, 128, 128, "bf16", 64),
        # trees of drafted tokens over ragged caches
        _step("step_trees", 16, 5000, True, 24, 16, 4, 128, 128, "bf16", 64),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _odd(rng, lo, hi):
    return _log_int(rng, lo, hi) | 1


def draw(rng):
    while True:
        case = _draw(rng)
        w = work(case)
        # below the largest listed cases (the plain form works on sequences of one length, filled up)
        limit = 3e10 if case.get("dtype") == "f32" else 2.7e11
        if w["bytes"] < 5e8 and w["flops"] < limit and _filled(case) < 2 ** 31:
            return case


def _filled(case):
    """Scores of the plain form."""
    if case["op"] == "prompt":
        lens = _lens(case["lens"])
        return len(lens) * case["heads"] * max(lens) * (max(lens) + case["before"])
    if case["op"] == "step":
        return case["requests"] * case["heads"] * case["drafts"] * (case["before"] + case["drafts"])
    return 0


def _draw(rng):
    op = rng.choice(("pages", "rotary", "rotary", "prompt", "prompt", "prompt", "step", "step", "step"))
    page = rng.choice((16, 16, 32, 64, 64, 128, 256))
    if op == "pages":
        requests = _log_int(rng, 1, 256)
        form = rng.choice(("step", "drafts", "prompts"))
        if form == "prompts":
            new = ",".join(str(rng.choice((0, 1, _log_int(rng, 2, 2000), _log_int(rng, 2, 2000)))) for _ in range(min(requests, 24)))
            return _pages(None, len(new.split(",")), _log_int(rng, 1, 4000), rng.choice((0, 3)), new, page,
                          rng.random() < 0.3)
        drafts = 1 if form == "step" else rng.randint(2, 64)
        return _pages(None, requests, _log_int(rng, 1, 16000), drafts if form == "drafts" else 0,
                      "%dx%d" % (requests, drafts), page, rng.random() < 0.2)
    dtype = rng.choice(("bf16", "bf16", "f32"))
    kv_heads = rng.choice((1, 2, 2, 3, 4, 4, 8))
    heads = kv_heads * rng.choice((1, 1, 2, 3, 4, 4, 8))
    dk = rng.choice((32, 64, 64, 80, 96, 128, 128, 128, 192, 256, rng.randint(16, 256)))
    dv = rng.choice((dk, dk, dk, 64, 128, rng.randint(16, 256)))
    if op == "rotary":
        dk += dk % 2
        rot = rng.choice((dk, dk, dk, 2 * rng.randint(1, dk // 2)))
        return _rotary(None, rng.choice((_log_int(rng, 1, 256), _odd(rng, 1, 8192))), heads, kv_heads, dk, dv, rot,
                       rng.choice(("half", "half", "interleaved")), dtype, rng.random() < 0.5, _log_int(rng, 100, 4000000),
                       rng.choice((0, page)))
    if op == "prompt":
        form = rng.choice(("one", "ragged", "goes_on"))
        if form == "one":
            return _prompt(None, str(_odd(rng, 2, 8192)), 0, heads, kv_heads, dk, dv, dtype, 0)
        lens = ",".join(str(rng.choice((0, 1, _log_int(rng, 2, 2048), _log_int(rng, 2, 2048))))
                        for _ in range(rng.randint(2, 12)))
        if not any(_lens(lens)):
            lens = "1," + lens
        if form == "ragged":
            return _prompt(None, lens, 0, heads, kv_heads, dk, dv, dtype, 0)
        return _prompt(None, lens, _log_int(rng, 1, 12000), heads, kv_heads, dk, dv, dtype, page)
    return _step(None, _log_int(rng, 1, 128), _log_int(rng, 1, 65536), rng.random() < 0.7,
                 rng.choice((1, 1, rng.randint(2, 64))), heads, kv_heads, dk, dv, dtype, page)


def _lens(text):
    if "x" in text:
        n, t = text.split("x")
        return [int(t)] * int(n)
    return [int(t) for t in text.split(",")]


def _spread(case, n, longest):
    """n lengths from `longest` down to nothing, in an order of their own."""
    return [longest * ((i * 7919 + 3) % n + 1) // n for i in range(n)] if n > 1 else [longest]


def _sizes(case):
    """Rows and keys of each sequence of an attention case."""
    if case["op"] == "prompt":
        new = _lens(case["lens"])
        past = _spread(case, len(new), case["before"]) if case["before"] else [0] * len(new)
    else:
        new = [case["drafts"]] * case["requests"]
        past = _spread(case, len(new), case["before"]) if case["ragged"] else [case["before"]] * len(new)
    return new, [p + n for p, n in zip(past, new)]


def work(case):
    if case["op"] == "pages":
        new = _lens(case["new"])
        tables = sum(-(-n // case["page"]) for n in new)
        return {"bytes": 8 * sum(new) + 24 * len(new) + 16 * tables, "flops": sum(new)}
    es = 2 if case["dtype"] == "bf16" else 4
    h, hk, dk, dv = case["heads"], case["kv_heads"], case["dk"], case["dv"]
    if case["op"] == "rotary":
        n = case["tokens"]
        moved = h * dk + hk * dk + (hk * dv if case["cache"] else 0)
        return {"bytes": 2 * n * moved * es + 8 * n, "flops": 3 * n * (h + hk) * case["rot"]}
    new, keys = _sizes(case)
    pairs = sum(n * (k - n) + n * (n + 1) // 2 for n, k in zip(new, keys))
    return {"bytes": (sum(new) * h * (dk + dv) + sum(k for n, k in zip(new, keys) if n) * hk * (dk + dv)) * es,
            "flops": 2 * pairs * h * (dk + dv)}


def _randn(gen, *shape, scale=1.0):
    return torch.randn(*shape, device="cuda", generator=gen) * scale


def _int32(x):
    return torch.tensor(x, device="cuda", dtype=torch.int32)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return {"pages": _prepare_pages, "rotary": _prepare_rotary, "prompt": _prepare_attention,
            "step": _prepare_attention}[case["op"]](case, gen)


def _table(gen, lens, places, page, most, pages):
    """Pages of requests with these lengths, in the places given of a table, from a pool in no order: table, the list of
    the pool's pages (those in use first) and how many are in use."""
    free = torch.randperm(pages, device="cuda", generator=gen).to(torch.int32)
    need = torch.tensor([-(-n // page) for n in lens], device="cuda")
    owner = torch.arange(len(lens), device="cuda").repeat_interleave(need)
    first = need.cumsum(0) - need
    table = torch.full((len(places) + 3, most), -1, device="cuda", dtype=torch.int32)
    at = torch.arange(owner.numel(), device="cuda")
    table[places[owner], at - first[owner]] = free[at]
    return table, free, need.sum()


def _prepare_pages(case, gen):
    n, page, new = case["requests"], case["page"], _lens(case["new"])
    before = _spread(case, n, case["before"])
    s = {"case": case, "page": page, "tokens": sum(new)}
    most = -(-(case["before"] + max(new)) // page)
    used, wanted = (sum(-(-t // page) for t in lens) for lens in (before, [b + m for b, m in zip(before, new)]))
    pages = used + (wanted - used) // 2 + 1 if case["short"] else wanted + 17
    s["places"] = torch.randperm(n + 3, device="cuda", generator=gen)[:n]
    s["slot"] = s["places"].to(torch.int32)
    s["table"], s["free"], taken = _table(gen, before, s["places"], page, most, pages)
    s["taken"] = taken.to(torch.int32).reshape(1)
    s["lens"] = torch.zeros(n + 3, device="cuda", dtype=torch.int32)
    s["lens"][s["places"]] = _int32(before)
    back = (torch.rand(n, device="cuda", generator=gen) * (case["kept"] + 1)).long()
    s["kept"] = (torch.tensor(before, device="cuda") - back).clamp(min=0).to(torch.int32)
    s["offsets"] = torch.tensor([0] + new, device="cuda").cumsum(0)
    s["place"], s["position"] = (torch.empty(s["tokens"], device="cuda", dtype=torch.int32) for _ in range(2))
    s["admitted"] = torch.empty(n, device="cuda", dtype=torch.int32)
    s["offsets_arg"] = None if len(set(new)) == 1 else s["offsets"]
    if own:
        from paper_2407_10730_amd import seqmix
        s["handle"] = seqmix.CachePages(tokens=s["tokens"], seqs=n, slots=n + 3, page=page, max_pages=most, pages=pages)
    return s


def _frequencies(case):
    """Radians per position, in float64; `scaled`: slow ones of a model trained on 8192 positions are 8 times slower, with a
    passage between."""
    half = case["rot"] // 2
    f = 500000.0 ** -(torch.arange(half, dtype=torch.float64, device="cuda") / half)
    if not case["scaled"]:
        return f
    turns = 8192 * f / (2 * math.pi)
    part = ((turns - 1) / (4 - 1)).clamp(0, 1)
    return f * part + f / 8 * (1 - part)


def _prepare_rotary(case, gen):
    n, h, hk, dk, dv, dt = case["tokens"], case["heads"], case["kv_heads"], case["dk"], case["dv"], _DT[case["dtype"]]
    # q, k and v are columns of one tensor, as the projection leaves them
    qkv = _randn(gen, n, h * dk + hk * dk + hk * dv).to(dt)
    s = {"case": case, "amplitude": 1.1 if case["scaled"] else 1.0, "freqs": _frequencies(case)}
    s["q"], s["k"], s["v"] = (t.view(n, -1, d) for t, d in zip(qkv.split([h * dk, hk * dk, hk * dv], 1), (dk, dk, dv)))
    s["position"] = torch.randint(0, case["far"] + 1, (n,), device="cuda", generator=gen, dtype=torch.int32)
    s["q_out"] = torch.empty(n, h, dk, device="cuda", dtype=dt)
    s["k_out"] = s["place"] = s["k_cache"] = s["v_cache"] = None
    page = case["cache"]
    pages = -(-n // page) + 2 if page else 0
    if page:  # rows of the cache in no order, some tokens without one
        place = torch.randperm(pages * page, device="cuda", generator=gen)[:n]
        s["place"] = torch.where(torch.rand(n, device="cuda", generator=gen) < 0.02, -1, place).to(torch.int32)
        s["k_cache"] = _randn(gen, pages, page, hk, dk).to(dt)
        s["v_cache"] = _randn(gen, pages, page, hk, dv).to(dt)
    else:
        s["k_out"] = torch.empty(n, hk, dk, device="cuda", dtype=dt)
    if own:
        from paper_2407_10730_amd import seqmix
        s["handle"] = seqmix.Rotary(
            tokens=n, heads=h, kv_heads=hk, dk=dk, dv=dv, rot=case["rot"], layout=case["layout"], dtype=case["dtype"],
            amplitude=s["amplitude"], page=page, pages=pages, q_strides=s["q"].stride()[:2], k_strides=s["k"].stride()[:2],
            v_strides=s["v"].stride()[:2])
    return s


def _tree(gen, requests, drafts):
    """Bit i of token j: token j sees drafted token i, its ancestors and itself."""
    sees = torch.zeros(requests, drafts, drafts, device="cuda", dtype=torch.bool)
    pick = torch.rand(requests, drafts, device="cuda", generator=gen)
    for j in range(drafts):
        if j:
            parent = (pick[:, j] * j).long()
            sees[:, j] = sees[torch.arange(requests, device="cuda"), parent]
        sees[:, j, j] = True
    return (sees.long() << torch.arange(drafts, device="cuda")).sum(-1).reshape(-1)


def _prepare_attention(case, gen):
    h, hk, dk, dv, dt, page = case["heads"], case["kv_heads"], case["dk"], case["dv"], _DT[case["dtype"]], case["page"]
    new, keys = _sizes(case)
    n, m = sum(new), len(new)
    s = {"case": case, "new": new, "keys": keys, "scale": dk ** -0.5, "tokens": n}
    s["q"] = _randn(gen, n, h, dk, scale=1.5).to(dt)
    s["o"] = torch.empty(n, h, dv, device="cuda", dtype=dt)
    s["offsets"] = torch.tensor([0] + new, device="cuda").cumsum(0)
    s["offsets_arg"] = None if len(set(new)) == 1 else s["offsets"]
    s["lens"] = s["table"] = s["slot"] = s["tree"] = None
    pages = most = 0
    if page:
        pages, most = sum(-(-t // page) for t in keys) + 5, -(-max(keys) // page)
        s["places"] = torch.randperm(m + 3, device="cuda", generator=gen)[:m]
        s["slot"] = s["places"].to(torch.int32)
        s["table"] = _table(gen, keys, s["places"], page, most, pages)[0]
        s["lens"] = torch.zeros(m + 3, device="cuda", dtype=torch.int32)
        s["lens"][s["places"]] = _int32(keys)
        s["k"] = torch.empty(pages, page, hk, dk, device="cuda", dtype=dt).normal_(generator=gen)
        s["v"] = torch.empty(pages, page, hk, dv, device="cuda", dtype=dt).normal_(generator=gen)
    else:  # k and v are columns of one tensor
        kv = _randn(gen, n, hk * (dk + dv)).to(dt)
        s["k"], s["v"] = (t.view(n, hk, d) for t, d in zip(kv.split([hk * dk, hk * dv], 1), (dk, dv)))
    if case["op"] == "step" and case["drafts"] > 1:
        s["tree"] = _tree(gen, m, case["drafts"])
    if own:
        from paper_2407_10730_amd import seqmix
        where = dict(page=page, max_pages=most, pages=pages, slots=m + 3) if page else dict(
            k_strides=s["k"].stride()[:2], v_strides=s["v"].stride()[:2])
        s["handle"] = seqmix.SoftmaxAttention(tokens=n, seqs=m, heads=h, kv_heads=hk, dk=dk, dv=dv, dtype=case["dtype"],
                                              mask="causal" if s["tree"] is None else "tree", scale=s["scale"], **where)
    return s


def run(s):
    op = s["case"]["op"]
    if op == "pages":
        if own:
            s["handle"].run(s["kept"], s["lens"], s["table"], s["free"], s["taken"], s["place"], s["position"], s["admitted"],
                            offsets=s["offsets_arg"], slot_index=s["slot"])
        else:
            _plain_pages(s)
        return {n: s[n] for n in ("lens", "table", "free", "taken", "place", "position", "admitted")}
    if op == "rotary":
        if own:
            s["handle"].run(s["q"], s["k"], s["v"], s["position"], s["freqs"], s["q_out"], s["k_out"], s["k_cache"],
                            s["v_cache"], s["place"])
        else:
            _plain_rotary(s)
        return {n: s[n] for n in ("q_out", "k_out", "k_cache", "v_cache") if s[n] is not None}
    if own:
        s["handle"].run(s["q"], s["k"], s["v"], s["o"], offsets=s["offsets_arg"], slot_index=s["slot"], lens=s["lens"],
                        table=s["table"], tree=s["tree"])
    else:
        _plain_attention(s)
    return {"o": s["o"]}


def _ragged(count):
    """For each of sum(count) things in a row: its owner, and its number among the owner's."""
    owner = torch.arange(count.numel(), device="cuda").repeat_interleave(count)
    return owner, torch.arange(owner.numel(), device="cuda") - (count.cumsum(0) - count)[owner]


def _plain_pages(s):
    page, at = s["page"], s["places"]
    have, new = s["lens"][at].long(), s["offsets"][1:] - s["offsets"][:-1]
    kept = torch.minimum(s["kept"].long(), have).clamp(min=0)
    pages = lambda n: (n + page - 1) // page  # noqa: E731
    # pages that are not needed any more go back, in the order of the batch
    back = pages(have) - pages(kept)
    owner, number = _ragged(back)
    gone = s["table"][at[owner], pages(kept)[owner] + number]
    taken = s["taken"].long() - back.sum()
    s["free"][taken + torch.arange(gone.numel(), device="cuda")] = gone
    # those that are needed are taken, as long as they last
    grow = pages(kept + new) - pages(kept)
    room = pages(kept + new) <= s["table"].shape[1]
    fits = room & ((grow == 0) | (torch.where(room, grow, 0).cumsum(0) + taken <= s["free"].numel()))
    grow = torch.where(fits, grow, 0)
    owner, number = _ragged(grow)
    s["table"][at[owner], pages(kept)[owner] + number] = s["free"][taken + torch.arange(owner.numel(), device="cuda")]
    s["taken"].copy_(taken + grow.sum())
    s["lens"][at] = torch.where(fits, kept + new, kept).to(torch.int32)
    s["admitted"].copy_(torch.where(fits, s["slot"], -1))
    owner, number = _ragged(new)
    position = kept[owner] + number
    place = s["table"][at[owner], (position // page).clamp(max=s["table"].shape[1] - 1)].long() * page + position % page
    s["place"].copy_(torch.where(fits[owner], place, -1))
    s["position"].copy_(torch.where(fits[owner], position, 0))


def _plain_rotary(s):
    case, dt = s["case"], s["q"].dtype
    rot = case["rot"]
    angle = s["position"].double()[:, None] * s["freqs"]
    c, sn = ((f(angle) * s["amplitude"]).float()[:, None] for f in (torch.cos, torch.sin))

    def turned(x):
        x = x.float()
        y = x.clone()
        if case["layout"] == "half":
            a, b = x[..., :rot // 2], x[..., rot // 2:rot]
            y[..., :rot // 2], y[..., rot // 2:rot] = a * c - b * sn, b * c + a * sn
        else:
            a, b = x[..., 0:rot:2], x[..., 1:rot:2]
            y[..., 0:rot:2], y[..., 1:rot:2] = a * c - b * sn, b * c + a * sn
        return y.to(dt)

    s["q_out"].copy_(turned(s["q"]))
    if not case["cache"]:
        s["k_out"].copy_(turned(s["k"]))
        return
    on = s["place"] >= 0
    page, row = s["place"][on].long() // case["cache"], s["place"][on].long() % case["cache"]
    s["k_cache"][page, row] = turned(s["k"])[on]
    s["v_cache"][page, row] = s["v"][on]


def _plain_attention(s):
    """Sequences side by side, filled up to the longest; scores of all rows and keys at once."""
    case, m = s["case"], len(s["new"])
    h, hk, dk, dv, page = case["heads"], case["kv_heads"], case["dk"], case["dv"], case["page"]
    new = s["offsets"][1:] - s["offsets"][:-1]
    keys = s["lens"][s["places"]].long() if page else new
    rows, cols = torch.arange(max(s["new"]), device="cuda"), torch.arange(max(s["keys"]), device="cuda")
    on_row, on_col = rows < new[:, None], cols < keys[:, None]
    row_at = torch.where(on_row, s["offsets"][:-1, None] + rows, 0)
    if page:
        held = s["table"][s["places"]][:, cols // page].long()
        k, v = (t[torch.where(on_col, held, 0), cols % page] for t in (s["k"], s["v"]))
    else:
        col_at = torch.where(on_col, s["offsets"][:-1, None] + cols, 0)
        k, v = s["k"][col_at], s["v"][col_at]
    q = (s["q"][row_at].float() * s["scale"]).reshape(m, rows.numel(), hk, h // hk, dk).permute(0, 2, 3, 1, 4)
    k, v = k.float().permute(0, 2, 3, 1).contiguous(), v.float().transpose(1, 2).contiguous()
    p = torch.matmul(q.reshape(m, hk, -1, dk), k).view(m, hk, h // hk, rows.numel(), cols.numel())
    back = (keys - new)[:, None, None]  # keys before the sequence's own rows
    sees = cols - back <= rows[:, None]
    if s["tree"] is not None:
        own_key = (cols - back).clamp(0, 63)
        sees = (cols < back) | ((s["tree"][row_at][:, :, None] >> own_key) & 1).bool()
    sees = sees & on_col[:, None]
    p = p.masked_fill_(~sees[:, None, None], -math.inf)
    p = p.sub_(p.amax(-1, keepdim=True).clamp_(min=-1e30)).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(m, hk, -1, cols.numel()), v).view(m, hk, h // hk, rows.numel(), dv)
    o = torch.where(total > 0, o / total, 0.0).permute(0, 3, 1, 2, 4).reshape(m, rows.numel(), h, dv)
    s["o"].copy_(o[on_row])


def exact(case, seed):
    s = prepare(case, seed)
    return {"pages": _exact_pages, "rotary": _exact_rotary, "prompt": _exact_attention, "step": _exact_attention}[case["op"]](s)


def _exact_pages(s):
    """A list of the pool's pages and a list of pages for each request, token by token."""
    page, places, new = s["page"], s["places"].tolist(), _lens(s["case"]["new"])
    lens, table, pool, kept = s["lens"].tolist(), s["table"].tolist(), s["free"].tolist(), s["kept"].tolist()
    taken, most = int(s["taken"]), len(table[0])
    gone = []
    for i, at in enumerate(places):
        keep = max(0, min(kept[i], lens[at]))
        used = [j for j in range(most) if j * page < lens[at]]
        gone += [table[at][j] for j in used if j * page >= keep]
        lens[at] = keep
    taken -= len(gone)
    pool[taken:taken + len(gone)] = gone
    place, position, admitted, full = [], [], [], False
    for i, at in enumerate(places):
        have = [j for j in range(most + new[i]) if j * page < lens[at]]
        want = [j for j in range(len(have) + new[i]) if j * page < lens[at] + new[i]]
        more = want[len(have):]
        full = full or (0 < len(more) and len(want) <= most and taken + len(more) > len(pool))
        if more and (full or len(want) > most):
            place += [-1] * new[i]
            position += [0] * new[i]
            admitted.append(-1)
            continue
        for j in more:
            table[at][j] = pool[taken]
            taken += 1
        for t in range(lens[at], lens[at] + new[i]):
            place.append(table[at][t // page] * page + t % page)
            position.append(t)
        lens[at] += new[i]
        admitted.append(at)
    return {"lens": _int32(lens), "table": _int32(table), "free": _int32(pool), "taken": _int32([taken]), "place": _int32(place),
            "position": _int32(position), "admitted": _int32(admitted)}


def _exact_rotary(s):
    """Pairs as complex numbers, multiplied by exp(i angle)."""
    case = s["case"]
    r = case["rot"]
    factor = s["amplitude"] * torch.exp(1j * torch.outer(s["position"].to(torch.float64), s["freqs"]))

    def turned(x):
        y = x.to(torch.float64)
        head, rest = y[..., :r], y[..., r:]
        if case["layout"] == "half":
            z = torch.complex(*(t.contiguous() for t in head.chunk(2, -1))) * factor[:, None]
            head = torch.cat([z.real, z.imag], -1)
        else:
            z = torch.view_as_complex(head.contiguous().unflatten(-1, (-1, 2))) * factor[:, None]
            head = torch.view_as_real(z).flatten(-2)
        return torch.cat([head, rest], -1)

    if not case["cache"]:
        return {"q_out": turned(s["q"]), "k_out": turned(s["k"])}
    out = {"q_out": turned(s["q"]), "k_cache": s["k_cache"].double(), "v_cache": s["v_cache"].double()}
    on = (s["place"] >= 0).nonzero()[:, 0]
    at = s["place"][on].long()
    out["k_cache"].flatten(0, 1)[at] = turned(s["k"])[on]
    out["v_cache"].flatten(0, 1)[at] = s["v"][on].double()
    return out


def _exact_attention(s):
    """Sequence by sequence and head by head, with a logarithm of the sum for the softmax."""
    case = s["case"]
    if 2e-5 * case["heads"] * len(s["new"]) * 20 > 15:
        return None
    rep, page = case["heads"] // case["kv_heads"], case["page"]
    o = torch.zeros(s["tokens"], case["heads"], case["dv"], device="cuda", dtype=torch.float64)
    first = 0
    for i, (n, m) in enumerate(zip(s["new"], s["keys"])):
        if not n:
            continue
        rows = slice(first, first + n)
        if page:
            used = s["table"][s["places"][i]][:-(-m // page)].long()
            k, v = s["k"][used].flatten(0, 1)[:m], s["v"][used].flatten(0, 1)[:m]
        else:
            k, v = s["k"][rows], s["v"][rows]
        i_at, j_at = torch.arange(n, device="cuda")[:, None], torch.arange(m, device="cuda")[None] - (m - n)
        hidden = j_at > i_at
        if s["tree"] is not None:
            hidden = (j_at >= 0) & ((s["tree"][rows][:, None] >> j_at.clamp(min=0)) % 2 == 0)
        for head in range(case["heads"]):
            kk, vv = k[:, head // rep].double(), v[:, head // rep].double()
            score = torch.where(hidden, -math.inf, s["scale"] * (s["q"][rows, head].double() @ kk.t().contiguous()))
            o[rows, head] = (score - torch.logsumexp(score, -1, keepdim=True)).exp() @ vv
        first += n
    return {"o": o}
