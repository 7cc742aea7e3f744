"""The serving operators from their definitions, in 64 bits and plain loops (numpy): what the tests compare with."""
import math

import numpy as np

# unit roundoff of each type: half a unit in the last place, relative
UNIT = {"bf16": 2.0**-8, "fp16": 2.0**-11, "fp32": 2.0**-24, "e4m3": 2.0**-4}


def extend(new, seq, table, free, count, page, max_tokens, n_pages=None):
    n_pages = len(free) if n_pages is None else n_pages
    table, seq_out = table.copy(), seq.copy()
    room = table.shape[1] * page
    count = min(max(int(count), 0), len(free))
    pages = tokens = popped = 0
    start, status, slots, positions, requests = [0], [], [], [], []
    for r, (n, old) in enumerate(zip(new.tolist(), seq.tolist())):
        if n < 0 or old < 0 or old + n > room:
            status.append(1)
            start.append(start[-1])
            continue
        has = -(-old // page)
        need = -(-(old + n) // page) - has
        pages += need
        tokens += n
        code = 2 if need and pages > count else 3 if n and tokens > max_tokens else 0
        status.append(code)
        if code:
            start.append(start[-1])
            continue
        for j in range(has, has + need):
            table[r, j] = free[count - 1 - popped]
            popped += 1
        for p in range(old, old + n):
            number = int(table[r, p // page])
            slots.append(number * page + p % page if 0 <= number < n_pages else -1)
            positions.append(p)
            requests.append(r)
        seq_out[r] = old + n
        start.append(start[-1] + n)
    pad = max_tokens - len(slots)
    i32 = lambda x: np.array(x, dtype=np.int32)  # noqa: E731
    return {"query_start": i32(start), "slots": i32(slots + [-1] * pad), "positions": i32(positions + [0] * pad),
            "requests": i32(requests + [-1] * pad), "seq_lens": seq_out, "free_count": i32([count - popped]),
            "status": i32(status), "block_table": table}


def release(done, seq, table, free, count, page):
    free, seq_out = free.copy(), seq.copy()
    count = min(max(int(count), 0), len(free))
    for r in np.nonzero(done)[0]:
        length = min(max(int(seq[r]), 0), table.shape[1] * page)
        for j in range(-(-length // page)):
            if count < len(free):
                free[count] = table[r, j]
                count += 1
        seq_out[r] = 0
    return {"seq_lens": seq_out, "free_count": np.array([count], dtype=np.int32), "free_pages": free}


def rotate(x, positions, inv_freq, axes, pairs, scale=1.0, inverse=False):
    """x [tokens, heads, dim] in float64, positions [axes, tokens] integers; the angle is reduced exactly, in integers."""
    y = x.copy()
    half = len(inv_freq)
    for i in range(half):
        angle = np.array([math.fmod(int(p) * math.fmod(inv_freq[i], 2 * math.pi), 2 * math.pi) if abs(int(p)) < 2**20
                          else _far_angle(int(p), inv_freq[i]) for p in positions[axes[i]]])
        c, s = scale * np.cos(angle)[:, None], scale * np.sin(angle)[:, None] * (-1.0 if inverse else 1.0)
        a, b = (i, i + half) if pairs == "half" else (2 * i, 2 * i + 1)
        y[..., a] = x[..., a] * c - x[..., b] * s
        y[..., b] = x[..., a] * s + x[..., b] * c
    return y


def _far_angle(p, f):
    """p * f modulo a turn for large p, with f as the exact rational that its double is and pi to 60 digits."""
    from fractions import Fraction

    pi = Fraction(314159265358979323846264338327950288419716939937510582097494, 10**59)
    turns = Fraction(f) * p / (2 * pi)
    return float((turns - math.floor(turns)) * 2 * pi)


def rotate_bound(x, half, pairs, dtype, y, scale=1.0):
    """How far an element may be off: sincospi is within 2 units of 2^-24 of its value and its argument within one, the
    products and the sum round three times, all in units of the pair's size; then one rounding to the type."""
    size = np.zeros_like(x)
    for i in range(half):
        a, b = (i, i + half) if pairs == "half" else (2 * i, 2 * i + 1)
        size[..., a] = size[..., b] = np.abs(x[..., a]) + np.abs(x[..., b])
    return UNIT[dtype] * np.abs(y) * (1 + 2.0**-20) + 16 * 2.0**-24 * abs(scale) * size + 2.0**-133


def attend(q, k, v, table, lens, scale, window=0, softcap=0.0, page_limit=None):
    """q [requests, q_heads, dim], k and v [pages, page, heads, dim] in float64.  Returns out, lse and, for bounds, the
    largest sum of |products| of a score and the sum of p|v|."""
    n, heads, dim = q.shape
    pages, page, kv = k.shape[:3]
    out, lse = np.zeros((n, heads, dim)), np.full((n, heads), -np.inf)
    size, mass = np.zeros((n, heads)), np.zeros((n, heads, dim))
    for r in range(n):
        length = min(max(int(lens[r]), 0), table.shape[1] * page)
        low = max(0, length - window) if window else 0
        t = np.arange(low, length)
        number = table[r, t // page] if len(t) else t
        there = (number >= 0) & (number < pages)
        number, off = number[there], (t % page)[there]
        if not len(number):
            continue
        for h in range(heads):
            kk, vv = k[number, off, h * kv // heads], v[number, off, h * kv // heads]
            s = kk @ q[r, h] * scale
            size[r, h] = (np.abs(kk) @ np.abs(q[r, h])).max() * abs(scale)
            if softcap:
                s = softcap * np.tanh(s / softcap)
            top = s.max()
            p = np.exp(s - top)
            out[r, h] = p @ vv / p.sum()
            mass[r, h] = p @ np.abs(vv) / p.sum()
            lse[r, h] = top + np.log(p.sum())
    return out, lse, size, mass


def attend_bound(y, size, mass, dim, dtype):
    """A score's products are summed in 32 bits (dim roundings at the size of the sum of their magnitudes at most, the
    scale and the exponential a few more); p's error is the score's, once above and once below the division; p enters
    its product with v with 15 bits at least."""
    score = (dim + 16) * 2.0**-23 * np.maximum(size, 1.0)
    return UNIT[dtype] * np.abs(y) * 1.001 + (2 * score[..., None] + 2.0**-14) * mass + 2.0**-25, score + 2.0**-14
