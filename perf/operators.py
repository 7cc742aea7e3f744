"""The cases in which the serving operators (pages, rotary positions, paged cache, decode attention) are measured.

`run` computes a case in plain torch operations where `own` is false, and through `paper_2002_12798_b200.ops` where it is
true.  A case names its operator in "op":

  extend    block tables, slot map and positions of one step from the requests' lengths
  release   the pages of finished requests back to the free list
  rotate    rotary positions on q and k (backward: the gradients of q and k)
  append    rotate q and k of a fused projection, write k and v into the paged cache
  attend    one new token per request against the paged cache
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32, "e4m3": torch.float8_e4m3fn}
BYTES = {"bf16": 2, "fp16": 2, "fp32": 4, "e4m3": 1}
E4M3_MAX = 448.0


# ----------------------------------------------------------------------------------------------------------------------
# the cases
# ----------------------------------------------------------------------------------------------------------------------
def _attend(name, requests, longest, q_heads, kv_heads, head_dim, page, dtype, cache, layout="token", window=0, softcap=0.0, ragged=True):
    return {"name": name, "op": "attend", "requests": requests, "longest": longest, "q_heads": q_heads, "kv_heads": kv_heads,
            "head_dim": head_dim, "page": page, "dtype": dtype, "cache": cache, "layout": layout, "window": window,
            "softcap": softcap, "ragged": ragged}


def _rotate(name, tokens, q_heads, kv_heads, head_dim, rotary_dim, axes, pairs, dtype, backward):
    return {"name": name, "op": "rotate", "tokens": tokens, "q_heads": q_heads, "kv_heads": kv_heads, "head_dim": head_dim,
            "rotary_dim": rotary_dim, "axes": axes, "pairs": pairs, "dtype": dtype, "backward": backward}


def _append(name, tokens, padding, q_heads, kv_heads, head_dim, axes, page, pages, dtype, cache):
    return {"name": name, "op": "append", "tokens": tokens, "padding": padding, "q_heads": q_heads, "kv_heads": kv_heads,
            "head_dim": head_dim, "rotary_dim": head_dim, "axes": axes, "pairs": "half", "page": page, "pages": pages,
            "dtype": dtype, "cache": cache}


def _extend(name, requests, prefills, chunk, page, row_pages, padding):
    return {"name": name, "op": "extend", "requests": requests, "prefills": prefills, "chunk": chunk, "page": page,
            "row_pages": row_pages, "padding": padding}


def listed():
    return [
        # a decode step of a small batch: one token per request, latency is all there is
        _extend("extend_decode", 64, 0, 1, 16, 512, 0),
        # a step that mixes decoding requests with chunks of long prompts
        _extend("extend_prefill", 1024, 100, 2048, 32, 512, 37),
        # a large batch of which a third has finished
        {"name": "release_third", "op": "release", "requests": 1024, "page": 32, "row_pages": 512, "done": 0.33},
        # a prompt of images and text (time, height, width), the whole sequence at once
        _rotate("rotate_prefill_bf16", 8192, 32, 8, 128, 128, 3, "half", "bf16", False),
        # the training direction in single precision: odd token count, neighbouring pairs, part of the head rotated
        _rotate("rotate_backward_fp32", 2047, 16, 16, 80, 64, 3, "adjacent", "fp32", True),
        # one decode step of a small batch
        _append("append_decode_fp16", 16, 0, 32, 8, 128, 1, 16, 256, "fp16", "fp16"),
        # a prompt chunk with padding behind it (a captured graph of fixed size)
        _append("append_prefill_bf16", 4099, 29, 32, 8, 128, 3, 16, 512, "bf16", "bf16"),
        # a decode step into a cache of 8 bits
        _append("append_decode_e4m3", 128, 0, 32, 8, 128, 1, 64, 64, "bf16", "e4m3"),
        # one request at the beginning of a conversation: the smallest call
        _attend("attend_short", 1, 33, 32, 8, 128, 16, "bf16", "bf16", ragged=False),
        # one request with a long document behind it: all the work is along the cache
        _attend("attend_long", 1, 131009, 32, 8, 128, 64, "fp16", "fp16", layout="head", ragged=False),
        # a serving batch, every length different, some rows empty
        _attend("attend_batch_bf16", 32, 16384, 32, 8, 128, 16, "bf16", "bf16"),
        # a larger batch of shorter requests over a cache of 8 bits
        _attend("attend_batch_e4m3", 128, 4096, 64, 8, 128, 32, "bf16", "e4m3"),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["extend", "release", "rotate", "rotate", "append", "append", "attend", "attend", "attend", "attend"])
    if op == "extend":
        requests = _log(rng, 1, 2000)
        prefills = rng.choice([0, rng.randint(0, requests // 8)])
        return {**_extend("", requests, prefills, _log(rng, 1, 2048), rng.choice([1, 8, 16, 24, 32, 64]), 512, rng.randint(0, 64)), "name": "drawn"}
    if op == "release":
        return {"name": "drawn", "op": "release", "requests": _log(rng, 1, 2000), "page": rng.choice([8, 16, 24, 32, 64]),
                "row_pages": 512, "done": rng.choice([0.02, 0.2, 0.6])}
    kv_heads = rng.choice([1, 2, 4, 8])
    group = rng.choice([1, 2, 4, 7, 8, 16])
    if op == "rotate":
        head_dim = rng.choice([64, 80, 96, 128, 256])
        rotary = rng.choice([head_dim, head_dim, head_dim // 2])
        dtype = rng.choice(["bf16", "fp16", "fp32"])
        tokens = _log(rng, 1, max(2, 40_000_000 // (kv_heads * (group + 1) * head_dim * BYTES[dtype] // 2)))
        return {**_rotate("", min(tokens, 16384), kv_heads * group, kv_heads, head_dim, rotary, rng.choice([1, 2, 3]), rng.choice(["half", "adjacent"]), dtype,
                          rng.random() < 0.5), "name": "drawn"}
    if op == "append":
        head_dim = rng.choice([64, 96, 128, 256])
        cache = rng.choice(["bf16", "fp16", "e4m3"])
        dtype = rng.choice(["bf16", "fp16"]) if cache == "e4m3" else cache
        tokens = _log(rng, 1, 4096) if cache != "e4m3" else _log(rng, 1, 512)
        page = rng.choice([8, 16, 24, 32, 64])
        return {**_append("", tokens, rng.choice([0, tokens // 7]), kv_heads * group, kv_heads, head_dim, rng.choice([1, 3]), page,
                          tokens // page + 2 + rng.randint(0, 100), dtype, cache), "name": "drawn"}
    head_dim = rng.choice([64, 80, 96, 128, 128, 256])
    cache = rng.choice(["bf16", "fp16", "e4m3"])
    dtype = rng.choice(["bf16", "fp16"]) if cache == "e4m3" else cache
    requests = _log(rng, 1, 256)
    most = 500_000_000 // (requests * 2 * kv_heads * head_dim * BYTES[cache])
    longest = _log(rng, 1, max(2, min(131072, most)))
    return {**_attend("", requests, longest, kv_heads * group, kv_heads, head_dim, rng.choice([8, 16, 24, 32, 64, 128]), dtype, cache,
                      rng.choice(["token", "head"]), rng.choice([0, 0, 0, max(1, longest // 3)]), rng.choice([0.0, 0.0, 0.0, 30.0]),
                      rng.random() < 0.8), "name": "drawn"}


# ----------------------------------------------------------------------------------------------------------------------
# what a program has in hand
# ----------------------------------------------------------------------------------------------------------------------
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 7919 + 12798)
    return g


def _normal(g, shape, dtype, spread=1.0):
    x = torch.randn(shape, generator=g, device="cuda", dtype=torch.float32 if dtype == torch.float32 else torch.bfloat16)
    return (x * spread).to(dtype)


def _integers(g, low, high, n):
    return torch.randint(low, high, (n,), generator=g, device="cuda", dtype=torch.int32)


def _frequencies(rotary_dim):
    return [10000.0 ** (-2.0 * i / rotary_dim) for i in range(rotary_dim // 2)]


def _axis_of_pairs(case):
    """Pairs in consecutive sections, one per axis: a quarter to the first axis, the rest shared evenly."""
    n, axes = case["rotary_dim"] // 2, case["axes"]
    if axes == 1:
        return [0] * n
    first = n // 4
    return [0] * first + [1 + (i * (axes - 1)) // (n - first) for i in range(n - first)]


def _positions(g, case, tokens):
    """Text runs along all axes at once; in a picture time stands still while height and width walk over its patches."""
    base = int(torch.randint(0, 4000, (1,), generator=g, device="cuda"))
    t = torch.arange(tokens, device="cuda", dtype=torch.int32)
    rows = [base + t // 9, base + (t // 32) % 48, base + t % 32][: case["axes"]] if case["axes"] > 1 else [base + t]
    return torch.stack(rows).to(torch.int32).contiguous()


def _table(case, positions):
    """cos and sin of every position that occurs, in 64 bits, rounded once."""
    f = torch.tensor(_frequencies(case["rotary_dim"]), device="cuda", dtype=torch.float64)
    angle = torch.arange(int(positions.max()) + 1, device="cuda", dtype=torch.float64)[:, None] * f
    return angle.cos().float(), angle.sin().float()


def _lengths(g, case):
    n = case["requests"]
    if not case["ragged"]:
        return torch.full((n,), case["longest"], device="cuda", dtype=torch.int32)
    lens = torch.randint(1, case["longest"] + 1, (n,), generator=g, device="cuda", dtype=torch.int32)
    lens[0] = case["longest"]
    if n >= 16:
        lens[n // 2] = 0
    return lens


def _cache(g, pages, case):
    """K and V as [pages, page, heads, dim]; with layout "head" the memory holds a head's tokens of a page side by side."""
    def one():
        if case.get("layout") == "head":
            x = _normal(g, (pages, case["kv_heads"], case["page"], case["head_dim"]), TYPES[case["cache"]]).transpose(1, 2)
        else:
            x = _normal(g, (pages, case["page"], case["kv_heads"], case["head_dim"]), TYPES[case["cache"]])
        return x

    return one(), one()


def _most_tokens(case):
    """Room for a step's tokens: a prompt chunk is half its largest size on average."""
    return case["requests"] + case["prefills"] * case["chunk"] * 5 // 8 + case["padding"]


def _inputs(case, seed):
    g = _generator(seed)
    op = case["op"]
    if op in ("extend", "release"):
        n, page, row = case["requests"], case["page"], case["row_pages"]
        seq = _integers(g, 0, row * page * 3 // 4, n)
        have = (seq + page - 1) // page
        pool = n * row
        order = torch.randperm(pool, generator=g, device="cuda").to(torch.int32)
        table = torch.where(torch.arange(row, device="cuda", dtype=torch.int32)[None] < have[:, None], order.view(n, row), torch.full_like(order.view(n, row), -1))
        free = torch.randperm(pool, generator=g, device="cuda").to(torch.int32)
        s = {"seq_lens": seq, "block_table": table.contiguous(), "free_pages": free, "page": page}
        if op == "release":
            s["done"] = torch.rand(n, generator=g, device="cuda") < case["done"]
            s["free_count"] = torch.zeros(1, device="cuda", dtype=torch.int32)
            return s
        new = torch.ones(n, device="cuda", dtype=torch.int32)
        new[_integers(g, 0, n, max(1, n // 16)).long()] = 0
        if case["prefills"]:
            at = torch.randperm(n, generator=g, device="cuda")[: case["prefills"]]
            new[at] = _integers(g, 1, case["chunk"] + 1, case["prefills"])
        s["new_lens"] = new
        s["max_tokens"] = _most_tokens(case)
        s["free_count"] = torch.full((1,), pool * 3 // 4, device="cuda", dtype=torch.int32)
        return s
    if op == "rotate":
        dtype = TYPES[case["dtype"]]
        pos = _positions(g, case, case["tokens"])
        q = _normal(g, (case["tokens"], case["q_heads"], case["head_dim"]), dtype)
        k = _normal(g, (case["tokens"], case["kv_heads"], case["head_dim"]), dtype)
        return {"q": q, "k": k, "positions": pos}
    if op == "append":
        dtype, d = TYPES[case["dtype"]], case["head_dim"]
        nq, nk, tokens = case["q_heads"], case["kv_heads"], case["tokens"]
        qkv = _normal(g, (tokens, (nq + 2 * nk) * d), dtype)
        pos = _positions(g, case, tokens)
        slots = torch.randperm(case["pages"] * case["page"], generator=g, device="cuda")[:tokens].to(torch.int32)
        if case["padding"]:
            slots[tokens - case["padding"]:] = -1
        k, v = _cache(g, case["pages"] + 1, case)  # the last page takes the padding's rows in the plain form
        return {"q": qkv[:, : nq * d].view(tokens, nq, d), "k": qkv[:, nq * d : (nq + nk) * d].view(tokens, nk, d),
                "v": qkv[:, (nq + nk) * d :].view(tokens, nk, d), "positions": pos, "slots": slots, "k_cache": k, "v_cache": v,
                "k_scale": 1.0 / 64 if case["cache"] == "e4m3" else 1.0, "v_scale": 1.0 / 64 if case["cache"] == "e4m3" else 1.0}
    lens = _lengths(g, case)
    row = -(-case["longest"] // case["page"])
    pages = int(((lens.long() + case["page"] - 1) // case["page"]).sum()) + 3
    have = (lens + case["page"] - 1) // case["page"]
    start = torch.cumsum(have, 0) - have
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    j = torch.arange(row, device="cuda")[None]
    table = torch.where(j < have[:, None], order[(start[:, None] + j).clamp(max=pages - 1)], torch.full_like(j.to(torch.int32), -1))
    k, v = _cache(g, pages, case)
    q = _normal(g, (case["requests"], case["q_heads"], case["head_dim"]), TYPES[case["dtype"]], 2.0)
    return {"q": q, "block_table": table.to(torch.int32).contiguous(), "seq_lens": lens, "k_cache": k, "v_cache": v,
            "k_scale": 0.75 if case["cache"] == "e4m3" else 1.0, "v_scale": 1.25 if case["cache"] == "e4m3" else 1.0}


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if case["op"] in ("rotate", "append"):
        s["cos"], s["sin"] = _table(case, s["positions"])
        s["axis"] = torch.tensor(_axis_of_pairs(case), device="cuda")
    if own:
        from paper_2002_12798_b200 import ops

        if case["op"] in ("rotate", "append"):
            s["rope"] = ops.RopePlan(case["head_dim"], case["rotary_dim"], inv_freq=_frequencies(case["rotary_dim"]),
                                     axes=_axis_of_pairs(case), pairs=case["pairs"])
        if case["op"] == "append":
            s["cache"] = ops.PagedCache(s["k_cache"][:-1], s["v_cache"][:-1], k_scale=s["k_scale"], v_scale=s["v_scale"])
        if case["op"] == "attend":
            s["cache"] = ops.PagedCache(s["k_cache"], s["v_cache"], k_scale=s["k_scale"], v_scale=s["v_scale"])
            s["plan"] = ops.AttendPlan(case["requests"], case["q_heads"], case["kv_heads"], case["head_dim"],
                                       window=case["window"], softcap=case["softcap"])
    return s


# ----------------------------------------------------------------------------------------------------------------------
# the plain forms
# ----------------------------------------------------------------------------------------------------------------------
def _plain_extend(s):
    new, old, table, free, count, page = s["new_lens"], s["seq_lens"], s["block_table"], s["free_pages"], s["free_count"], s["page"]
    n, row = table.shape
    fits = (new >= 0) & (old >= 0) & (old.long() + new <= row * page)
    want = torch.where(fits, new, 0)
    have = (old + page - 1) // page
    need = (old + want + page - 1) // page - have
    pages_to, tokens_to = torch.cumsum(need, 0), torch.cumsum(want, 0)
    paged, roomy = (need == 0) | (pages_to <= count), (want == 0) | (tokens_to <= s["max_tokens"])
    status = torch.where(~fits, 1, torch.where(~paged, 2, torch.where(~roomy, 3, 0)))
    granted = torch.where(status == 0, want, 0)
    need = torch.where(status == 0, need, 0)
    first = torch.cumsum(need, 0) - need
    start = torch.cat([torch.zeros(1, dtype=torch.int64, device=new.device), torch.cumsum(granted, 0)])
    i = torch.arange(s["max_tokens"], device=new.device)
    r = torch.searchsorted(start[1:], i, right=True).clamp(max=n - 1)
    live = i < start[-1]
    position = old[r] + i - start[r]
    j = position // page
    j_all = torch.arange(row, device=new.device)[None]
    fresh = (j_all >= have[:, None]) & (j_all < (have + need)[:, None])
    taken = (count - 1 - (first[:, None] + j_all - have[:, None])).clamp(0, free.numel() - 1)
    table = torch.where(fresh, free[taken], table)
    slot = table[r, j.clamp(max=row - 1)] * page + position % page
    whole = lambda x: x.to(torch.int32)  # noqa: E731
    return {"query_start": whole(start), "slots": whole(torch.where(live, slot, -1)), "positions": whole(torch.where(live, position, 0)),
            "requests": whole(torch.where(live, r, -1)), "seq_lens": whole(old + granted), "free_count": whole(count - need.sum()),
            "status": whole(status), "block_table": table}


def _plain_release(s):
    old, table, free, count, page = s["seq_lens"], s["block_table"], s["free_pages"], s["free_count"], s["page"]
    back = torch.where(s["done"], (old + page - 1) // page, 0)
    to = torch.cumsum(back, 0)
    at = torch.arange(free.numel(), device=free.device) - count
    r = torch.searchsorted(to, at, right=True).clamp(max=old.numel() - 1)
    j = (at - (to[r] - back[r])).clamp(0, table.shape[1] - 1)
    free = torch.where((at >= 0) & (at < to[-1]), table[r, j], free)
    return {"seq_lens": torch.where(s["done"], 0, old), "free_count": (count + to[-1]).to(torch.int32), "free_pages": free}


def _plain_rotate(s, x, sign):
    case = s["case"]
    half = case["rotary_dim"] // 2
    at = s["positions"].long()[s["axis"]].T  # [tokens, pairs]
    pair = torch.arange(half, device=x.device)
    cos, sin = s["cos"][at, pair][:, None], sign * s["sin"][at, pair][:, None]
    x = x.float()
    if case["pairs"] == "half":
        a, b = x[..., :half], x[..., half : 2 * half]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    else:
        a, b = x[..., 0 : 2 * half : 2], x[..., 1 : 2 * half : 2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    return torch.cat([turned, x[..., 2 * half :]], -1)


def _plain_store(cache, slots, rows, scale):
    flat = cache.view(-1, *cache.shape[2:])
    rows = rows / scale
    if cache.dtype == torch.float8_e4m3fn:
        rows = rows.clamp(-E4M3_MAX, E4M3_MAX).to(cache.dtype)
        flat.view(torch.uint8)[slots] = rows.view(torch.uint8)
    else:
        flat[slots] = rows.to(cache.dtype)


def _plain_append(s):
    slots = torch.where(s["slots"] < 0, (s["k_cache"].shape[0] - 1) * s["case"]["page"], s["slots"]).long()
    _plain_store(s["k_cache"], slots, _plain_rotate(s, s["k"], 1.0), s["k_scale"])
    _plain_store(s["v_cache"], slots, s["v"].float(), s["v_scale"])
    return _plain_rotate(s, s["q"], 1.0).to(s["q"].dtype)


def _pages(cache, pages):
    """The pages named in a block table, in 32 bits: [requests, tokens, heads, dim]."""
    if cache.dtype == torch.float8_e4m3fn:
        return cache.view(torch.uint8)[pages].view(cache.dtype).flatten(1, 2).float()
    return cache[pages].flatten(1, 2).float()


def _plain_attend(s):
    case, q, lens = s["case"], s["q"], s["seq_lens"]
    n, heads, d = case["requests"], case["kv_heads"], case["head_dim"]
    pages = s["block_table"].clamp(min=0).long()
    t = torch.arange(pages.shape[1] * case["page"], device=q.device)[None]
    live = t < lens[:, None]
    if case["window"]:
        live = live & (t >= (lens - case["window"])[:, None])
    live = live[:, None, None]
    k = _pages(s["k_cache"], pages) * s["k_scale"]
    logits = q.float().view(n, heads, -1, d) @ k.permute(0, 2, 3, 1) / math.sqrt(d)
    del k
    if case["softcap"]:
        logits = case["softcap"] * torch.tanh(logits / case["softcap"])
    logits = torch.where(live, logits, -torch.inf)
    top = logits.amax(-1, keepdim=True)
    top = torch.where(top == -torch.inf, 0.0, top)
    p = torch.exp(logits - top)
    total = p.sum(-1, keepdim=True)
    v = _pages(s["v_cache"], pages) * s["v_scale"]
    o = p @ v.permute(0, 2, 1, 3) / torch.where(total == 0, 1.0, total)
    lse = torch.where(total == 0, -torch.inf, top + torch.log(total))
    return {"out": o.reshape(q.shape).to(q.dtype), "lse": lse.reshape(n, -1)}


def _held(s, q):
    """q and the caches; what is held in 8 bits as the values it stands for."""
    k, v = s["k_cache"][:-1], s["v_cache"][:-1]
    if k.dtype == torch.float8_e4m3fn:
        k, v = k.to(torch.bfloat16), v.to(torch.bfloat16)
    return {"q": q, "k_cache": k, "v_cache": v}


def run(state):
    case = state["case"]
    op = case["op"]
    if not own:
        if op == "extend":
            return _plain_extend(state)
        if op == "release":
            return _plain_release(state)
        if op == "rotate":
            sign = -1.0 if case["backward"] else 1.0
            dtype = state["q"].dtype
            return {"q": _plain_rotate(state, state["q"], sign).to(dtype), "k": _plain_rotate(state, state["k"], sign).to(dtype)}
        if op == "append":
            return _held(state, _plain_append(state))
        return _plain_attend(state)
    from paper_2002_12798_b200 import ops

    if op == "extend":
        step = ops.pages_extend(state["new_lens"], state["seq_lens"], state["block_table"], state["free_pages"],
                                state["free_count"], state["page"], state["max_tokens"])
        return {"query_start": step.query_start, "slots": step.slots, "positions": step.positions, "requests": step.requests,
                "seq_lens": step.seq_lens, "free_count": step.free_count, "status": step.status, "block_table": state["block_table"]}
    if op == "release":
        seq_lens, free_count = ops.pages_release(state["done"], state["seq_lens"], state["block_table"], state["free_pages"],
                                                 state["free_count"], state["page"])
        return {"seq_lens": seq_lens, "free_count": free_count, "free_pages": state["free_pages"]}
    if op == "rotate":
        q, k = state["rope"].rotate([state["q"], state["k"]], state["positions"], inverse=case["backward"])
        return {"q": q, "k": k}
    if op == "append":
        q = state["rope"].append(state["q"], state["k"], state["v"], state["positions"], state["slots"], state["cache"])
        return _held(state, q)
    out, lse = state["plan"].attend(state["q"], state["cache"], state["block_table"], state["seq_lens"], return_lse=True)
    return {"out": out, "lse": lse}


# ----------------------------------------------------------------------------------------------------------------------
# what a pass cannot do without, and what it should give
# ----------------------------------------------------------------------------------------------------------------------
def work(case):
    op = case["op"]
    if op == "extend":
        fresh = (case["requests"] + case["prefills"] * case["chunk"] // 2) // case["page"]
        return {"bytes": 20 * case["requests"] + 12 * _most_tokens(case) + 8 * fresh, "flops": 0}
    if op == "release":
        return {"bytes": case["requests"] * (9 + case["done"] * 8 * case["row_pages"] * 3 // 8), "flops": 0}
    width = case["head_dim"] * BYTES[case["dtype"]]
    if op == "rotate":
        rows = case["tokens"] * (case["q_heads"] + case["kv_heads"])
        return {"bytes": 2 * rows * width + 4 * case["axes"] * case["tokens"], "flops": 3 * rows * case["rotary_dim"]}
    if op == "append":
        live = case["tokens"] - case["padding"]
        moved = 2 * case["tokens"] * case["q_heads"] * width + 2 * live * case["kv_heads"] * (width + case["head_dim"] * BYTES[case["cache"]])
        return {"bytes": moved + (4 + 4 * case["axes"]) * case["tokens"], "flops": 3 * case["tokens"] * (case["q_heads"] + case["kv_heads"]) * case["rotary_dim"]}
    mean = case["longest"] / 2 if case["ragged"] and case["requests"] > 1 else case["longest"]
    tokens = case["requests"] * (min(mean, case["window"]) if case["window"] else mean)
    held = 2 * tokens * case["kv_heads"] * case["head_dim"] * BYTES[case["cache"]]
    return {"bytes": held + case["requests"] * case["q_heads"] * (2 * width + 4) + 4 * tokens / case["page"], "flops": 4 * tokens * case["q_heads"] * case["head_dim"]}


def _turned(case, x, positions, sign):
    """A pair as a complex number, times exp(i angle)."""
    half = case["rotary_dim"] // 2
    f = torch.tensor(_frequencies(case["rotary_dim"]), dtype=torch.float64, device=x.device)
    angle = torch.empty(x.shape[0], half, dtype=torch.float64, device=x.device)
    for i, a in enumerate(_axis_of_pairs(case)):
        angle[:, i] = sign * positions[a].double() * f[i]
    wave = torch.polar(torch.ones_like(angle), angle)[:, None]
    y = x.double().clone()
    if case["pairs"] == "half":
        z = torch.complex(y[..., :half], y[..., half : 2 * half]) * wave
        y[..., :half], y[..., half : 2 * half] = z.real, z.imag
    else:
        z = torch.complex(y[..., 0 : 2 * half : 2], y[..., 1 : 2 * half : 2]) * wave
        y[..., 0 : 2 * half : 2], y[..., 1 : 2 * half : 2] = z.real, z.imag
    return y


def exact(case, seed):
    op = case["op"]
    if op in ("extend", "release"):
        return None  # whole numbers: equal or wrong
    s = _inputs(case, seed)
    if op == "rotate":
        sign = -1.0 if case["backward"] else 1.0
        return {"q": _turned(case, s["q"], s["positions"], sign), "k": _turned(case, s["k"], s["positions"], sign)}
    if op == "append":
        kept = s["slots"] >= 0
        at = s["slots"][kept].long()
        got = {"q": _turned(case, s["q"], s["positions"], 1.0)}
        for name, rows, scale in (("k_cache", _turned(case, s["k"], s["positions"], 1.0), s["k_scale"]), ("v_cache", s["v"].double(), s["v_scale"])):
            held = s[name][:-1].double().contiguous()
            rows = rows / scale
            if case["cache"] == "e4m3":
                rows = rows.clamp(-E4M3_MAX, E4M3_MAX)
            held.view(-1, *held.shape[2:])[at] = rows[kept]
            got[name] = held
        return got
    n, heads, d = case["requests"], case["kv_heads"], case["head_dim"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full((n, case["q_heads"]), -math.inf, dtype=torch.float64, device="cuda")
    for r, length in enumerate(s["seq_lens"].tolist()):
        low = max(0, length - case["window"]) if case["window"] else 0
        if low >= length:
            continue
        t = torch.arange(low, length, device="cuda")
        page, slot = s["block_table"][r].long()[t // case["page"]], t % case["page"]
        for h in range(heads):
            group = slice(h * case["q_heads"] // heads, (h + 1) * case["q_heads"] // heads)
            k = s["k_cache"].view(torch.uint8 if case["cache"] == "e4m3" else s["k_cache"].dtype)[page, slot, h].view(s["k_cache"].dtype).double() * s["k_scale"]
            v = s["v_cache"].view(torch.uint8 if case["cache"] == "e4m3" else s["v_cache"].dtype)[page, slot, h].view(s["v_cache"].dtype).double() * s["v_scale"]
            x = s["q"][r, group].double() @ k.T / math.sqrt(d)
            if case["softcap"]:
                x = case["softcap"] * torch.tanh(x / case["softcap"])
            lse[r, group] = torch.logsumexp(x, -1)
            out[r, group] = torch.softmax(x, -1) @ v
    return {"out": out, "lse": lse}
