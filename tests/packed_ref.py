"""The cache of 4 bits and sampling from their definitions, in 64 bits (numpy): what the tests compare with."""
import numpy as np


def bf16_down(x):
    """The largest bf16 number that is not above x."""
    _, e = np.frexp(x)
    unit = np.ldexp(1.0, np.maximum(e, -125) - 8)  # a bf16 number has 8 bits, its smallest step is 2^-133
    y = np.floor(x / unit) * unit
    return np.where(y < -((2 - 2.0**-7) * 2.0**127), -np.inf, y)


def bf16_near(x):
    """x rounded to fp32 and that to bf16, both to nearest even."""
    with np.errstate(over="ignore"):
        bits = np.asarray(x, dtype=np.float64).astype(np.float32).view(np.uint32).astype(np.uint64)
    bits = ((bits + 0x7FFF + ((bits >> 16) & 1)) >> 16) << 16
    return bits.astype(np.uint32).view(np.float32).astype(np.float64)


def quantise(x, group):
    """x [..., dim] in float64 -> (codes [..., dim], low, step [..., dim / group]); a group that does not have finite numbers for all
    of them has low NaN."""
    x = x.reshape(*x.shape[:-1], -1, group)
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        finite = np.isfinite(x).all(-1)
        x = np.where(finite[..., None], x, 0.0)
        low = bf16_down(x.min(-1))
        step = bf16_near((x.max(-1) - low) / 15)
        good = finite & np.isfinite(low) & np.isfinite(step)
        low, step = np.where(good, low, np.nan), np.where(good, step, 0.0)
        code = np.rint((x - low[..., None]) / step[..., None])
    code = np.where(step[..., None] > 0, np.minimum(code, 15), 0.0)
    return code.reshape(*code.shape[:-2], -1).astype(np.int64), low, step


def values(codes, low, step):
    """In 32 bits, as a cache gives them back before the last rounding."""
    g = codes.reshape(*codes.shape[:-1], low.shape[-1], -1)
    with np.errstate(invalid="ignore"):
        y = (low[..., None] + step[..., None] * g).astype(np.float32)
    return y.reshape(codes.shape).astype(np.float64)


def held(x, group):
    """What the cache holds for x, in 64 bits."""
    codes, low, step = quantise(x, group)
    g = codes.reshape(*codes.shape[:-1], low.shape[-1], -1)
    return (low[..., None] + step[..., None] * g).reshape(codes.shape)


def sample(x, u, temperature, top_k, top_p, min_p):
    """One row: (token, log of its probability, distance of u from the nearest border that decides, in probability)."""
    x = np.where(np.isnan(x), -np.inf, x.astype(np.float64))
    if x.max() == -np.inf:
        return -1, -np.inf, 1.0
    order = np.lexsort((np.arange(len(x)), -x))
    if not temperature > 0:
        return int(order[0]), 0.0, 1.0
    top = x[order[0]]
    w = (x[order] == np.inf).astype(np.float64) if top == np.inf else np.exp((x[order] - top) / temperature)
    kept = np.ones(len(x), dtype=bool) if top_k <= 0 else np.arange(len(x)) < top_k
    kept &= w >= min(min_p, 1.0)
    n = int(kept.sum())  # a beginning of the order
    if top_p < 1:
        ahead = np.cumsum(w[:n]) - w[:n]
        n = max(1, int((ahead < top_p * w[:n].sum()).sum()))
    by = np.argsort(order[:n])
    at, w = order[:n][by], w[:n][by]
    upto = np.cumsum(w)
    target = min(max(float(u), 0.0), 1 - 2.0**-24) * upto[-1]
    i = min(int(np.searchsorted(upto, target, side="right")), n - 1)
    return int(at[i]), float(np.log(w[i] / upto[-1])), float(np.abs(upto - target).min() / upto[-1])


def attend(q, k, v, at, scale, softcap=0.0):
    """One request: q [q_heads, dim], k and v (codes, low, step) of all slots [slots, heads, ..], at: the slots that take part, in
    float64.  Returns out, lse and bounds for their errors before the last rounding of out."""
    heads, dim = q.shape
    kv = k[0].shape[1]
    if not len(at):
        return np.zeros((heads, dim)), np.full(heads, -np.inf), np.zeros((heads, dim)), np.zeros(heads)

    def parts(x, h):  # values, and the sizes of what they are made of
        codes, low, step = (y[at, h] for y in x)
        g = codes.reshape(len(at), low.shape[-1], -1)
        return (low[..., None] + step[..., None] * g).reshape(len(at), -1), (np.abs(low)[..., None] + step[..., None] * g).reshape(len(at), -1)

    out, lse, out_bound, lse_bound = np.zeros((heads, dim)), np.zeros(heads), np.zeros((heads, dim)), np.zeros(heads)
    for h in range(heads):
        (kk, ka), (vv, va) = parts(k, h * kv // heads), parts(v, h * kv // heads)
        s = kk @ q[h] * scale
        # the products' sum has dim roundings at its terms' size, q's smallest elements lose 2^-36 of the largest, the groups'
        # sums, the scale and the exponential a few more
        size = (ka @ np.abs(q[h])).max() * abs(scale)
        off = (dim + 24) * 2.0**-23 * max(size, 1.0) + 2.0**-36 * dim * np.abs(q[h]).max() * ka.max() * abs(scale)
        if softcap:
            s = softcap * np.tanh(s / softcap)
            off += 2.0**-19 * min(softcap, np.abs(s).max() + 1)
        top = s.max()
        p = np.exp(s - top)
        lse[h] = top + np.log(p.sum())
        p /= p.sum()
        out[h] = p @ vv
        # weights: the score's error, above and below the division; two terms of 11 bits, sums of 32 over the tokens (the
        # matrix unit cuts off rather than rounds: one step each); what is 2^-24 of the largest weight loses 2^-40 of that
        weight = np.maximum(np.abs(v[1][at, h * kv // heads]).max(-1), v[2][at, h * kv // heads].max(-1))
        out_bound[h] = (2 * off + 2.0**-20 + (np.log2(len(at)) + 40) * 2.0**-23) * (p @ va) + 15 * len(at) ** 0.5 * 2.0**-33 * (p * weight).max()
        lse_bound[h] = off + 2.0**-21 + 2.0**-22 * abs(lse[h])
    return out, lse, out_bound, lse_bound
