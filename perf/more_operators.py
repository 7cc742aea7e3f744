"""The cases in which the cache of 4 bits (written, read back, attended to) and sampling are measured.

`run` computes a case in plain torch operations where `own` is false, and through `paper_2002_12798_b200.ops` where it is
true.  A case names its operator in "op":

  append    rotate q and k of a fused projection, quantise k and v into the paged cache as they are written, and read the
            written tokens back
  read      tokens of many requests out of the cache, in 16 bits
  attend    one new token per request against the cache
  sample    a token per row of logits: temperature, top-k, min-p, top-p, from given uniform numbers

A group of `group` elements of a head is held as codes of 4 bits and two numbers in bf16:
  low = its smallest element, rounded down;  step = (its largest element - low) / 15, rounded to nearest;
  code = (element - low) / step, rounded to nearest even and clamped to 0 .. 15 (0 where step is 0);
a code stands for low + step * code.  k is quantised as the exact rotation gives it, in 64 bits here, because values next to
the border between two codes are common.
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
BYTES = {"bf16": 2, "fp16": 2, "fp32": 4}


# ----------------------------------------------------------------------------------------------------------------------
# the cases
# ----------------------------------------------------------------------------------------------------------------------
def _append(name, tokens, padding, q_heads, kv_heads, head_dim, group, axes, pairs, page, dtype):
    return {"name": name, "op": "append", "tokens": tokens, "padding": padding, "q_heads": q_heads, "kv_heads": kv_heads, "head_dim": head_dim,
            "group": group, "axes": axes, "pairs": pairs, "page": page, "pages": tokens // page + 8, "dtype": dtype}


def _read(name, tokens, kv_heads, head_dim, group, page, dtype):
    return {"name": name, "op": "read", "tokens": tokens, "kv_heads": kv_heads, "head_dim": head_dim, "group": group, "page": page, "dtype": dtype}


def _attend(name, requests, longest, q_heads, kv_heads, head_dim, group, page, dtype, window=0, softcap=0.0, ragged=True):
    return {"name": name, "op": "attend", "requests": requests, "longest": longest, "q_heads": q_heads, "kv_heads": kv_heads, "head_dim": head_dim,
            "group": group, "page": page, "dtype": dtype, "window": window, "softcap": softcap, "ragged": ragged}


def _sample(name, rows, vocab, dtype, spread, top_k, top_p, min_p, mixed=False):
    """spread: standard deviation of the logits.  mixed: every row has settings of its own, some rows are greedy."""
    return {"name": name, "op": "sample", "rows": rows, "vocab": vocab, "dtype": dtype, "spread": spread, "top_k": top_k, "top_p": top_p,
            "min_p": min_p, "mixed": mixed}


def listed():
    return [
        # a decode step of a batch: latency is all there is
        _append("append_decode", 64, 0, 32, 8, 128, 64, 1, "half", 16, "bf16"),
        # a prompt chunk of images and text with padding behind it (a captured graph of fixed size)
        _append("append_prefill", 4099, 29, 32, 8, 128, 64, 3, "half", 16, "bf16"),
        # a short conversation comes back for another turn
        _read("read_short", 700, 8, 128, 64, 16, "bf16"),
        # the contexts of a batch, to be attended to by a prompt chunk or sent to another machine
        _read("read_contexts", 65537, 8, 128, 32, 64, "fp16"),
        # one request at the beginning of a conversation: the smallest call
        _attend("attend_short", 1, 33, 32, 8, 128, 64, 16, "bf16", ragged=False),
        # one request with a long document behind it: all the work is along the cache
        _attend("attend_long", 1, 131009, 32, 8, 128, 32, 64, "fp16", ragged=False),
        # a serving batch, every length different, some rows empty
        _attend("attend_batch", 64, 16384, 32, 8, 128, 64, 16, "bf16"),
        # a larger batch of shorter requests, 16 q heads to a cache head
        _attend("attend_wide", 128, 4096, 64, 4, 128, 64, 32, "fp16"),
        # one conversation: the usual settings, latency is all there is
        _sample("sample_one", 1, 32000, "fp32", 3.0, 50, 0.95, 0.0),
        # a batch whose head gives 16 bits, nucleus sampling over an odd vocabulary
        _sample("sample_nucleus", 64, 100003, "bf16", 2.5, 0, 0.9, 0.0),
        # rollouts for training: the model's own distribution, nothing cut off
        _sample("sample_whole", 128, 131072, "fp32", 2.0, 0, 1.0, 0.0),
        # a large serving batch, settings by request
        _sample("sample_mixed", 256, 150001, "bf16", 3.0, 40, 0.9, 0.05, mixed=True),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["append", "append", "read", "attend", "attend", "attend", "sample", "sample", "sample"])
    if op == "sample":
        dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
        vocab = _log(rng, 1000, 260000)
        rows = _log(rng, 1, min(512, 75_000_000 // (vocab * BYTES[dtype])))
        return {**_sample("", rows, vocab, dtype, rng.choice([1.0, 2.0, 3.0, 4.0]), rng.choice([0, 0, 1, 20, 50, 200]), rng.choice([1.0, 0.5, 0.9, 0.95]),
                          rng.choice([0.0, 0.0, 0.02, 0.1]), rng.random() < 0.4), "name": "drawn"}
    kv_heads = rng.choice([1, 2, 4, 8])
    head_dim = rng.choice([64, 96, 128, 128, 256])
    group = 32 if head_dim == 96 else rng.choice([32, 64])
    page = rng.choice([16, 32, 48, 64, 128])
    dtype = rng.choice(["bf16", "fp16"])
    if op == "read":
        most = 65537 * 8 * 128 // (kv_heads * head_dim)
        return {**_read("", _log(rng, 1, min(100_000, most)), kv_heads, head_dim, group, page, dtype), "name": "drawn"}
    q_heads = kv_heads * rng.choice([1, 2, 4, 7, 8, 16])
    if op == "append":
        tokens = _log(rng, 1, 4099)
        return {**_append("", tokens, rng.choice([0, tokens // 7]), q_heads, kv_heads, head_dim, group, rng.choice([1, 3]), rng.choice(["half", "half", "adjacent"]),
                          page, dtype), "name": "drawn"}
    requests = _log(rng, 1, 256)
    most = 1_000_000_000 // (requests * 2 * kv_heads * head_dim)
    longest = _log(rng, 1, max(2, min(131072, most)))
    return {**_attend("", requests, longest, q_heads, kv_heads, head_dim, group, page, dtype, rng.choice([0, 0, 0, max(1, longest // 3)]),
                      rng.choice([0.0, 0.0, 0.0, 30.0]), rng.random() < 0.8), "name": "drawn"}


# ----------------------------------------------------------------------------------------------------------------------
# what a program has in hand
# ----------------------------------------------------------------------------------------------------------------------
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 6700417 + 2002)
    return g


def _normal(g, shape, dtype, spread=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * spread).to(dtype)


def _frequencies(head_dim):
    return [10000.0 ** (-2.0 * i / head_dim) for i in range(head_dim // 2)]


def _axis_of_pairs(case):
    """Pairs in consecutive sections, one per axis: a quarter to the first axis, the rest shared evenly."""
    n, axes = case["head_dim"] // 2, case["axes"]
    if axes == 1:
        return [0] * n
    first = n // 4
    return [0] * first + [1 + (i * (axes - 1)) // (n - first) for i in range(n - first)]


def _positions(g, case):
    """Text runs along all axes at once; in a picture time stands still while height and width walk over its patches."""
    base = int(torch.randint(0, 4000, (1,), generator=g, device="cuda"))
    t = torch.arange(case["tokens"], device="cuda", dtype=torch.int32)
    rows = [base + t // 9, base + (t // 32) % 48, base + t % 32] if case["axes"] > 1 else [base + t]
    return torch.stack(rows).to(torch.int32).contiguous()


def _keys_and_values(g, case, tokens):
    """Keys have channels with an offset of their own, values tokens of different size."""
    shape = (tokens, case["kv_heads"], case["head_dim"])
    offset = torch.randn(shape[1:], generator=g, device="cuda") ** 3
    k = (torch.randn(shape, generator=g, device="cuda") + offset).to(TYPES[case["dtype"]])
    size = torch.exp(0.7 * torch.randn((tokens, 1, 1), generator=g, device="cuda"))
    v = (torch.randn(shape, generator=g, device="cuda") * size).to(TYPES[case["dtype"]])
    return k, v


def _chunks(total, tokens=65536):
    return [(a, min(a + tokens, total)) for a in range(0, total, tokens)]


def _lengths(g, case):
    n = case["requests"]
    if not case["ragged"]:
        return torch.full((n,), case["longest"], device="cuda", dtype=torch.int32)
    lens = torch.randint(1, case["longest"] + 1, (n,), generator=g, device="cuda", dtype=torch.int32)
    lens[0] = case["longest"]
    if n >= 16:
        lens[n // 2] = 0
    return lens


def _inputs(case, seed):
    """Everything but the cache's content, and a generator for that."""
    g = _generator(seed)
    op = case["op"]
    if op == "sample":
        n = case["rows"]
        s = {"logits": _normal(g, (n, case["vocab"]), TYPES[case["dtype"]], case["spread"]), "u": torch.rand(n, generator=g, device="cuda")}
        one = torch.ones(n, device="cuda")
        s["temperature"], s["top_k"] = 0.8 * one, torch.full((n,), case["top_k"], device="cuda", dtype=torch.int32)
        s["top_p"], s["min_p"] = case["top_p"] * one, case["min_p"] * one
        if case["mixed"]:
            kind = torch.randint(0, 4, (4, n), generator=g, device="cuda")
            s["temperature"] = torch.tensor([0.0, 0.6, 1.0, 1.3], device="cuda")[kind[0]]
            s["top_k"] = torch.tensor([0, 0, 1, 3], device="cuda", dtype=torch.int32)[kind[1]] * case["top_k"]
            s["top_p"] = torch.where(kind[2] < 2, s["top_p"], one)
            s["min_p"] = torch.where(kind[3] < 1, s["min_p"], torch.zeros_like(one))
        return s, g
    if op == "append":
        dtype, d, tokens = TYPES[case["dtype"]], case["head_dim"], case["tokens"]
        nq, nk = case["q_heads"], case["kv_heads"]
        k, v = _keys_and_values(g, case, tokens)
        qkv = torch.cat([_normal(g, (tokens, nq, d), dtype), k, v], 1).view(tokens, -1)
        slots = torch.randperm(case["pages"] * case["page"], generator=g, device="cuda")[:tokens].to(torch.int32)
        if tokens >= 256:  # a chunk of a prompt lies in whole pages
            pages = torch.randperm(case["pages"], generator=g, device="cuda")
            t = torch.arange(tokens, device="cuda")
            slots = (pages[t // case["page"]] * case["page"] + t % case["page"]).to(torch.int32)
        if case["padding"]:
            slots[tokens - case["padding"]:] = -1
        return {"q": qkv[:, : nq * d].view(tokens, nq, d), "k": qkv[:, nq * d : (nq + nk) * d].view(tokens, nk, d),
                "v": qkv[:, (nq + nk) * d :].view(tokens, nk, d), "positions": _positions(g, case), "slots": slots}, g
    if op == "read":
        pages = case["tokens"] // case["page"] + 3
        order = torch.randperm(pages, generator=g, device="cuda")
        t = torch.arange(case["tokens"], device="cuda")
        return {"slots": (order[t // case["page"]] * case["page"] + t % case["page"]).to(torch.int32), "pages": pages}, g
    lens = _lengths(g, case)
    row = -(-case["longest"] // case["page"])
    have = (lens + case["page"] - 1) // case["page"]
    pages = int(have.sum()) + 3
    start = torch.cumsum(have, 0) - have
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    j = torch.arange(row, device="cuda")[None]
    table = torch.where(j < have[:, None], order[(start[:, None] + j).clamp(max=pages - 1)], torch.full_like(j.to(torch.int32), -1))
    q = _normal(g, (case["requests"], case["q_heads"], case["head_dim"]), TYPES[case["dtype"]])
    return {"q": q, "block_table": table.to(torch.int32).contiguous(), "seq_lens": lens, "pages": pages}, g


def prepare(case, seed):
    s, g = _inputs(case, seed)
    s["case"] = case
    op = case["op"]
    if op == "sample":
        return s
    d, heads, group = case["head_dim"], case["kv_heads"], case["group"]
    if op == "append":
        f = torch.tensor(_frequencies(d), device="cuda", dtype=torch.float64)
        angle = torch.arange(int(s["positions"].max()) + 1, device="cuda", dtype=torch.float64)[:, None] * f
        s["cos"], s["sin"], s["axis"] = angle.cos(), angle.sin(), torch.tensor(_axis_of_pairs(case), device="cuda")
    pages = s.get("pages", case.get("pages"))
    total = pages * case["page"]
    if own:
        from paper_2002_12798_b200 import ops

        s["cache"] = ops.PackedCache.zeros(pages, case["page"], heads, d, group=group)
        if op == "append":
            s["rope"] = ops.RopePlan(d, inv_freq=_frequencies(d), axes=_axis_of_pairs(case), pairs=case["pairs"])
        if op == "attend":
            s["plan"] = ops.AttendPlan(case["requests"], case["q_heads"], heads, d, window=case["window"], softcap=case["softcap"])
    else:
        for name in ("k", "v"):
            s[name + "_codes"] = torch.zeros(total, heads, d, device="cuda", dtype=torch.uint8)
            for part in ("_low", "_step"):
                s[name + part] = torch.zeros(total, heads, d // group, device="cuda", dtype=torch.bfloat16)
    if op == "append":
        return s
    for a, b in _chunks(total):  # what earlier steps have put there
        k, v = _keys_and_values(g, case, b - a)
        if own:
            s["cache"].write(k, v, torch.arange(a, b, device="cuda", dtype=torch.int32))
        else:
            for name, x in (("k", k), ("v", v)):
                s[name + "_codes"][a:b], s[name + "_low"][a:b], s[name + "_step"][a:b] = _quantised(x.double(), group)
    return s


# ----------------------------------------------------------------------------------------------------------------------
# the plain forms
# ----------------------------------------------------------------------------------------------------------------------
def _down(x):
    """The largest bf16 number that is not above x (64 bits)."""
    near = x.float().to(torch.bfloat16)
    bits = near.view(torch.int16)
    below = torch.where(near == 0, -32767, torch.where(bits > 0, bits - 1, bits + 1)).to(torch.int16).view(torch.bfloat16)
    return torch.where(near.double() > x, below, near)


def _quantised(x, group):
    x = x.unflatten(-1, (-1, group))
    low = _down(x.amin(-1))
    step = ((x.amax(-1) - low.double()) / 15).float().to(torch.bfloat16)
    code = torch.round((x - low.double()[..., None]) / step.double()[..., None]).clamp(0, 15)
    code = torch.where(step[..., None] == 0, torch.zeros_like(code), code)
    return code.to(torch.uint8).flatten(-2), low, step


def _values(codes, low, step):
    group = codes.shape[-1] // low.shape[-1]
    return (low.float()[..., None] + step.float()[..., None] * codes.unflatten(-1, (-1, group)).float()).flatten(-2)


def _plain_rotate(s, x):
    case, half = s["case"], s["case"]["head_dim"] // 2
    at = s["positions"].long()[s["axis"]].T  # [tokens, pairs]
    pair = torch.arange(half, device=x.device)
    cos, sin = s["cos"][at, pair][:, None].to(x.dtype), s["sin"][at, pair][:, None].to(x.dtype)
    a, b = (x[..., :half], x[..., half:]) if case["pairs"] == "half" else (x[..., 0::2], x[..., 1::2])
    turned = [a * cos - b * sin, b * cos + a * sin]
    return torch.cat(turned, -1) if case["pairs"] == "half" else torch.stack(turned, -1).flatten(-2)


def _plain_read(s, slots):
    there = (slots >= 0)[:, None, None]
    at = slots.clamp(min=0).long()
    dtype = TYPES[s["case"]["dtype"]]
    return {x: torch.where(there, _values(s[x + "_codes"][at], s[x + "_low"][at], s[x + "_step"][at]), 0.0).to(dtype) for x in ("k", "v")}


def _plain_append(s):
    case = s["case"]
    q = _plain_rotate(s, s["q"].float()).to(s["q"].dtype)
    live = case["tokens"] - case["padding"]
    slots = s["slots"][:live].long()
    for name, x in (("k", _plain_rotate(s, s["k"].double())), ("v", s["v"].double())):
        s[name + "_codes"][slots], s[name + "_low"][slots], s[name + "_step"][slots] = _quantised(x[:live], case["group"])
    return {"q": q, **_plain_read(s, s["slots"])}


def _plain_attend(s):
    case, q, lens = s["case"], s["q"], s["seq_lens"]
    n, heads, d, page = case["requests"], case["kv_heads"], case["head_dim"], case["page"]
    t = torch.arange(s["block_table"].shape[1] * page, device=q.device)
    at = s["block_table"].clamp(min=0).long()[:, t // page] * page + t % page
    t = t[None]
    live = t < lens[:, None]
    if case["window"]:
        live = live & (t >= (lens - case["window"])[:, None])
    live = live[:, None, None]
    k = _values(s["k_codes"][at], s["k_low"][at], s["k_step"][at])
    logits = q.float().view(n, heads, -1, d) @ k.permute(0, 2, 3, 1) / math.sqrt(d)
    del k
    if case["softcap"]:
        logits = case["softcap"] * torch.tanh(logits / case["softcap"])
    logits = torch.where(live, logits, -torch.inf)
    top = logits.amax(-1, keepdim=True)
    top = torch.where(top == -torch.inf, 0.0, top)
    p = torch.exp(logits - top)
    total = p.sum(-1, keepdim=True)
    v = _values(s["v_codes"][at], s["v_low"][at], s["v_step"][at])
    o = p @ v.permute(0, 2, 1, 3) / torch.where(total == 0, 1.0, total)
    lse = torch.where(total == 0, -torch.inf, top + torch.log(total))
    return {"out": o.reshape(q.shape).to(q.dtype), "lse": lse.reshape(n, -1)}


def _plain_sample(s):
    """In 64 bits: a uniform number next to the border between two tokens decides which one it is."""
    x, vocab = s["logits"], s["logits"].shape[1]
    # by value, ties in the order of their index
    value, index = torch.sort(x, dim=1, descending=True, stable=True)
    t = s["temperature"].double()[:, None]
    greedy = t <= 0
    w = torch.exp((value.double() - value[:, :1].double()) / torch.where(greedy, 1.0, t))
    rank = torch.arange(vocab, device=x.device)[None]
    k = s["top_k"].long()[:, None]
    kept = ((k <= 0) | (rank < k)) & (w >= s["min_p"].double()[:, None])
    w = torch.where(kept, w, 0.0)
    ahead = torch.cumsum(w, 1) - w
    kept = kept & ((ahead < s["top_p"].double()[:, None] * w.sum(1, keepdim=True)) | (rank == 0))
    kept = torch.where(greedy, rank == 0, kept)
    w = torch.where(kept, w, 0.0)
    weight = torch.zeros_like(w).scatter_(1, index, w)  # in the order of the tokens again
    upto = torch.cumsum(weight, 1)
    mass = upto[:, -1:]
    past = (upto > s["u"].double()[:, None] * mass) & (weight > 0)
    token = past.to(torch.uint8).argmax(1)
    return {"token": token.to(torch.int32), "logprob": torch.log(weight.gather(1, token[:, None]) / mass)[:, 0].float()}


def run(state):
    case = state["case"]
    op = case["op"]
    if not own:
        if op == "append":
            return _plain_append(state)
        if op == "read":
            return _plain_read(state, state["slots"])
        return _plain_attend(state) if op == "attend" else _plain_sample(state)
    if op == "append":
        q = state["rope"].append(state["q"], state["k"], state["v"], state["positions"], state["slots"], state["cache"])
        k, v = state["cache"].read(state["slots"], dtype=q.dtype)
        return {"q": q, "k": k, "v": v}
    if op == "read":
        k, v = state["cache"].read(state["slots"], dtype=TYPES[case["dtype"]])
        return {"k": k, "v": v}
    if op == "attend":
        out, lse = state["plan"].attend(state["q"], state["cache"], state["block_table"], state["seq_lens"], return_lse=True)
        return {"out": out, "lse": lse}
    from paper_2002_12798_b200 import ops

    token, logprob = ops.sample(state["logits"], state["u"], temperature=state["temperature"], top_k=state["top_k"], top_p=state["top_p"],
                                min_p=state["min_p"], return_logprob=True)
    return {"token": token, "logprob": logprob}


# ----------------------------------------------------------------------------------------------------------------------
# what a pass cannot do without, and what it should give
# ----------------------------------------------------------------------------------------------------------------------
def work(case):
    op = case["op"]
    if op == "sample":
        n = case["rows"] * case["vocab"]
        return {"bytes": n * BYTES[case["dtype"]] + 28 * case["rows"], "flops": 2 * n}
    d, heads = case["head_dim"], case["kv_heads"]
    held = 2 * heads * (d // 2 + 4 * d // case["group"])  # a token of the cache
    wide = heads * d * BYTES[case["dtype"]]
    if op == "read":
        return {"bytes": case["tokens"] * (held + 2 * wide + 4), "flops": 4 * case["tokens"] * heads * d}
    if op == "append":
        live, q = case["tokens"] - case["padding"], case["q_heads"] * d * BYTES[case["dtype"]]
        return {"bytes": case["tokens"] * (2 * q + 8 + 4 * case["axes"] + 2 * wide) + live * (2 * wide + 2 * held),
                "flops": case["tokens"] * d * (3 * case["q_heads"] + 15 * heads)}
    mean = case["longest"] / 2 if case["ragged"] and case["requests"] > 1 else case["longest"]
    tokens = case["requests"] * (min(mean, case["window"]) if case["window"] else mean)
    rows = case["requests"] * case["q_heads"]
    return {"bytes": tokens * held + rows * (2 * d * BYTES[case["dtype"]] + 4) + 4 * tokens / case["page"], "flops": 4 * tokens * case["q_heads"] * d}


def _held(x, group):
    """What a cache of 4 bits gives back for x, in 64 bits: the grid of 16 values, and the nearest."""
    x = x.double().reshape(*x.shape[:-1], -1, group)
    lo = x.min(-1, keepdim=True).values
    # rounded down to 8 bits: to a multiple of 2^(exponent - 8), where lo = mantissa * 2^exponent with a mantissa in [1/2, 1)
    _, exponent = torch.frexp(lo)
    unit = torch.ldexp(torch.ones_like(lo), exponent.clamp(min=-125) - 8)
    lo = torch.floor(lo / unit) * unit
    step = ((x.max(-1, keepdim=True).values - lo) / 15).to(torch.float32).to(torch.bfloat16).double()
    code = ((x - lo) / torch.where(step == 0, 1.0, step)).round().clamp(max=15.0)
    return (lo + code * step).flatten(-2)


def _turned(case, x, positions):
    """A pair as a complex number, times exp(i angle)."""
    half = case["head_dim"] // 2
    angle = torch.empty(x.shape[0], half, dtype=torch.float64, device=x.device)
    for i, (a, f) in enumerate(zip(_axis_of_pairs(case), _frequencies(case["head_dim"]))):
        angle[:, i] = positions[a].double() * f
    wave = torch.polar(torch.ones_like(angle), angle)[:, None]
    pair = x.double().unflatten(-1, (2, half)).transpose(-1, -2) if case["pairs"] == "half" else x.double().unflatten(-1, (half, 2))
    z = torch.view_as_real(torch.complex(pair[..., 0], pair[..., 1]) * wave)
    return (z.transpose(-1, -2) if case["pairs"] == "half" else z).flatten(-2)


def _exact_sample(s):
    """Row by row: the tokens in their order, one bound after the other, then along the row."""
    tokens, logprobs = [], []
    for r in range(s["logits"].shape[0]):
        x = s["logits"][r].double()
        t, k, p, least = (s[n][r].item() for n in ("temperature", "top_k", "top_p", "min_p"))
        order = torch.argsort(x, descending=True, stable=True)
        if t <= 0:
            tokens.append(order[0])
            logprobs.append(torch.zeros((), dtype=torch.float64, device="cuda"))
            continue
        order = order[:k] if k > 0 else order
        w = torch.exp((x[order] - x[order[0]]) / t)
        w = w[w >= least]
        n = max(1, int((torch.cumsum(w, 0) - w < p * w.sum()).sum()))
        at, by = torch.sort(order[:n])
        w = w[:n][by]
        upto = torch.cumsum(w, 0)
        i = min(int(torch.searchsorted(upto, s["u"][r].double() * upto[-1], right=True)), n - 1)
        tokens.append(at[i])
        logprobs.append(torch.log(w[i] / upto[-1]))
    return {"token": torch.stack(tokens).to(torch.int32), "logprob": torch.stack(logprobs)}


def exact(case, seed):
    s, g = _inputs(case, seed)
    op = case["op"]
    if op == "sample":
        return _exact_sample(s)
    group = case["group"]
    if op == "append":
        there = (s["slots"] >= 0)[:, None, None]
        k, v = _held(_turned(case, s["k"], s["positions"]), group), _held(s["v"], group)
        return {"q": _turned(case, s["q"], s["positions"]), "k": torch.where(there, k, 0.0), "v": torch.where(there, v, 0.0)}
    both = [_keys_and_values(g, case, b - a) for a, b in _chunks(s["pages"] * case["page"])]
    k, v = (torch.cat([x[i] for x in both]) for i in (0, 1))
    if op == "read":
        at = s["slots"].long()
        return {"k": _held(k[at], group), "v": _held(v[at], group)}
    heads, d = case["kv_heads"], case["head_dim"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(s["q"].shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    for r, length in enumerate(s["seq_lens"].tolist()):
        low = max(0, length - case["window"]) if case["window"] else 0
        if low >= length:
            continue
        t = torch.arange(low, length, device="cuda")
        at = s["block_table"][r].long()[t // case["page"]] * case["page"] + t % case["page"]
        for h in range(heads):
            of = slice(h * case["q_heads"] // heads, (h + 1) * case["q_heads"] // heads)
            x = s["q"][r, of].double() @ _held(k[at, h], group).T / math.sqrt(d)
            if case["softcap"]:
                x = case["softcap"] * torch.tanh(x / case["softcap"])
            lse[r, of] = torch.logsumexp(x, -1)
            out[r, of] = torch.softmax(x, -1) @ _held(v[at, h], group)
    return {"out": out, "lse": lse}
