"""A decoder layer's serving steps from end to end: pages, rotary positions, paged cache, decode attention.

    python examples/decode_step.py [--steps N] [--cache bf16|e4m3|4bit]

A prompt of every request goes into the cache in one step (its own attention is left to the caller's prefill kernel), then
tokens are generated one at a time: a step's `pages_extend`, `append`, `attend` and `sample` are captured in a CUDA graph once
and replayed, nothing is copied to the host in between.  Random projections stand in for the model; the last step is
checked against plain torch.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2002_12798_b200 import ops  # noqa: E402


def main():
    p = argparse.ArgumentParser()
    p.add_argument("--steps", type=int, default=20)
    p.add_argument("--cache", choices=["bf16", "e4m3", "4bit"], default="bf16")
    a = p.parse_args()
    torch.manual_seed(0)
    requests, q_heads, heads, dim, page, row = 8, 32, 8, 128, 16, 64
    pages, dev = requests * row, "cuda"
    int32 = dict(dtype=torch.int32, device=dev)

    # what a serving program keeps: the pool, the block table, a cache per layer (one here) and the plans
    table = torch.full((requests, row), -1, **int32)
    free = torch.randperm(pages, device=dev).to(torch.int32)
    free_count, seq_lens = torch.tensor([pages], **int32), torch.zeros(requests, **int32)
    held = torch.bfloat16 if a.cache == "bf16" else torch.float8_e4m3fn
    scale = 1.0 if a.cache == "bf16" else 1.0 / 64
    if a.cache == "4bit":
        cache = ops.PackedCache.zeros(pages, page, heads, dim)
    else:
        k_cache = torch.zeros(pages, page, heads, dim, device=dev).to(held)
        v_cache = torch.zeros(pages, page, heads, dim, device=dev).to(held)
        cache = ops.PagedCache(k_cache, v_cache, k_scale=scale, v_scale=scale)
    rope = ops.RopePlan(dim, sections=[16, 24, 24])  # time, height, width; text moves along all three
    attention = ops.AttendPlan(requests, q_heads, heads, dim)

    def split(x):  # a fused projection as q, k and v: views, no copies
        return (t.unflatten(1, (-1, dim)) for t in x.split([q_heads * dim, heads * dim, heads * dim], 1))

    # the prompts, all in one step
    prompt = torch.randint(1, 200, (requests,), **int32)
    prompt[3] = 0  # a row of the table that no request has yet
    room = requests * 200
    step = ops.pages_extend(prompt, seq_lens, table, free, free_count, page, room)
    q, k, v = split(torch.randn(room, (q_heads + 2 * heads) * dim, device=dev, dtype=torch.bfloat16))
    rope.append(q, k, v, step.positions.expand(3, -1), step.slots, cache)
    seq_lens.copy_(step.seq_lens)
    free_count.copy_(step.free_count)

    # decoding: one token per request that has begun
    new = (prompt > 0).to(torch.int32)
    fused = torch.empty(requests, (q_heads + 2 * heads) * dim, device=dev, dtype=torch.bfloat16)
    to_logits = torch.randn(q_heads * dim, 5000, device=dev, dtype=torch.bfloat16)
    uniforms = torch.empty(requests, device=dev)

    def decode():
        s = ops.pages_extend(new, seq_lens, table, free, free_count, page, requests)
        q, k, v = split(fused)
        q = rope.append(q, k, v, s.positions.expand(3, -1), s.slots, cache)
        rows = torch.zeros(requests + 1, q_heads, dim, device=dev, dtype=q.dtype)  # token -> its request's row
        rows[torch.where(s.requests < 0, requests, s.requests).long()] = q
        out = attention.attend(rows[:requests], cache, table, s.seq_lens)
        token = ops.sample(out.flatten(1) @ to_logits, uniforms, temperature=0.8, top_k=50, top_p=0.95)
        seq_lens.copy_(s.seq_lens)
        free_count.copy_(s.free_count)
        return rows, out, token

    before = seq_lens.clone(), free_count.clone(), table.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        fused.normal_()
        uniforms.uniform_()
        decode()  # warm-up
    torch.cuda.current_stream().wait_stream(side)
    for now, was in zip((seq_lens, free_count, table), before):
        now.copy_(was)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rows, out, token = decode()
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    start.record()
    for _ in range(a.steps):
        fused.normal_()
        uniforms.uniform_()
        graph.replay()
    end.record()
    torch.cuda.synchronize()

    # the last step again in plain torch
    worst = 0.0
    for r in range(requests):
        n = int(seq_lens[r])
        if n == 0:
            assert not out[r].any()
            continue
        t = torch.arange(n, device=dev)
        at, off = table[r, t // page].long(), t % page
        if a.cache == "4bit":
            kk, vv = cache.read((at * page + off).to(torch.int32), dtype=torch.float32)
        else:
            kk, vv = (c.view(torch.uint8 if a.cache == "e4m3" else held)[at, off].view(held).float() * scale for c in (k_cache, v_cache))
        x = torch.einsum("hgd,thd->hgt", rows[r].float().view(heads, -1, dim), kk) * dim**-0.5
        want = torch.einsum("hgt,thd->hgd", torch.softmax(x, -1), vv).reshape(q_heads, dim)
        worst = max(worst, float((out[r].float() - want).abs().max() / want.abs().max()))
    assert worst < 0.01 and not attention.failed(), worst
    assert ((token >= 0) & (token < 5000)).all()
    done = torch.ones(requests, dtype=torch.bool, device=dev)
    seq_lens, free_count = ops.pages_release(done, seq_lens, table, free, free_count, page)
    assert int(free_count) == pages and sorted(free.tolist()) == list(range(pages))
    print("%d decoding steps of %d requests (%s cache): %.1f us a step, largest error %.4f of the output's size"
          % (a.steps, requests, a.cache, start.elapsed_time(end) / a.steps * 1e3, worst))


if __name__ == "__main__":
    main()
