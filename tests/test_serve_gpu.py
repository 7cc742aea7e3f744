"""The serving operators on the GPU against their definitions in 64 bits, at the sizes, masks and layouts where they can
go wrong."""
import math

import numpy as np
import pytest

import serve_ref as ref

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32, "e4m3": torch.float8_e4m3fn}


@pytest.fixture(scope="module")
def ops():
    from paper_2002_12798_b200 import ops

    return ops


def f64(t):
    return t.to(torch.float32).cpu().double().numpy()


def cuda(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


# ----------------------------------------------------------------------------------------------------------------------
# pages
# ----------------------------------------------------------------------------------------------------------------------
def pool(r, requests, row, page, spare):
    """lengths, a table that holds their pages and a free stack, all page numbers distinct"""
    seq = r.integers(0, row * page + 1, requests).astype(np.int32)
    have = -(-seq // page)
    numbers = r.permutation(int(have.sum()) + spare).astype(np.int32)
    table = np.full((requests, row), -7, dtype=np.int32)
    at = 0
    for i, n in enumerate(have):
        table[i, :n] = numbers[at : at + n]
        at += n
    free = np.full(len(numbers), -9, dtype=np.int32)
    free[:spare] = numbers[at:]
    return seq, table, free


def check_extend(ops, new, seq, table, free, count, page, max_tokens, wide=0):
    want = ref.extend(new, seq, table, free, count, page, max_tokens)
    n, row = table.shape
    held = np.full((n, row + wide), 77, dtype=np.int32)
    held[:, :row] = table
    held = cuda(held)
    args = [cuda(new), cuda(seq), held[:, :row], cuda(free), cuda(np.array([count], dtype=np.int32))]
    for _ in range(2):  # the inputs are unchanged: the same call gives the same answer
        step = ops.pages_extend(*args, page, max_tokens)
        for name in step._fields:
            assert np.array_equal(getattr(step, name).cpu().numpy(), want[name]), name
        assert np.array_equal(held[:, :row].cpu().numpy(), want["block_table"])
        assert (held[:, row:] == 77).all()
    assert np.array_equal(args[1].cpu().numpy(), seq) and int(args[4]) == count
    return step


@pytest.mark.parametrize("page", [1, 3, 16])
@pytest.mark.parametrize("requests", [1, 5, 255, 1024, 1025, 2500])
def test_extend(ops, requests, page):
    r = np.random.default_rng(requests * 31 + page)
    seq, table, free = pool(r, requests, 40, page, 6 * requests)
    seq = (seq * 0.6).astype(np.int32)
    new = r.integers(0, 5, requests).astype(np.int32)
    new[r.integers(0, requests, max(1, requests // 9))] = 30
    total = int(new.sum())
    check_extend(ops, new, seq, table, free, 6 * requests, page, total + 11, wide=3)


@pytest.mark.parametrize("short", ["pages", "tokens", "both"])
def test_extend_refuses_what_does_not_fit_and_only_that(ops, short):
    r = np.random.default_rng(len(short))
    seq, table, free = pool(r, 1300, 20, 4, 900)
    new = r.integers(0, 9, 1300).astype(np.int32)
    new[[3, 700]] = -1
    seq[[4, 1100]] = -2
    new[5] = 2**31 - 1
    count, tokens = (400 if short != "tokens" else 900), (900 if short != "pages" else 20000)
    step = check_extend(ops, new, seq, table, free, count, 4, tokens)
    status = step.status.cpu().numpy()
    assert set(status) >= {0, 1} | {"pages": {2}, "tokens": {3}, "both": {2, 3}}[short]


def test_extend_of_nothing_and_of_one_token(ops):
    zero, table = np.zeros(3, dtype=np.int32), np.full((3, 2), -1, dtype=np.int32)
    check_extend(ops, zero, zero, table, np.array([5, 6], dtype=np.int32), 2, 8, 4)
    check_extend(ops, np.array([0, 1, 0], dtype=np.int32), zero, table, np.array([1, 0], dtype=np.int32), 2, 8, 1)
    check_extend(ops, np.array([0, 1, 0], dtype=np.int32), zero, table, np.array([1, 0], dtype=np.int32), 0, 8, 1)


def test_extend_gives_a_foreign_page_no_slot(ops):
    table = np.array([[99, -1]], dtype=np.int32)  # the request's own page number is not one of the pool
    check_extend(ops, np.array([6], dtype=np.int32), np.array([3], dtype=np.int32), table, np.array([0, 1, 1], dtype=np.int32), 2, 4, 8)
    # a free count that is no count is clamped
    check_extend(ops, np.array([6], dtype=np.int32), np.array([0], dtype=np.int32), table, np.array([0, 1, 1], dtype=np.int32), -5, 4, 8)


@pytest.mark.parametrize("requests,page", [(1, 1), (7, 16), (1024, 3), (2100, 5)])
@pytest.mark.parametrize("share", [0.0, 0.3, 1.0])
def test_release(ops, requests, page, share):
    r = np.random.default_rng(requests + page)
    seq, table, free = pool(r, requests, 33, page, 5)
    done = r.random(requests) < share
    want = ref.release(done, seq, table, free, 5, page)
    got_free = cuda(free)
    seq_out, count_out = ops.pages_release(cuda(done), cuda(seq), cuda(table), got_free, cuda(np.array([5], dtype=np.int32)), page)
    assert np.array_equal(seq_out.cpu().numpy(), want["seq_lens"])
    assert np.array_equal(count_out.cpu().numpy(), want["free_count"])
    assert np.array_equal(got_free.cpu().numpy(), want["free_pages"])


def test_release_drops_what_the_stack_has_no_room_for(ops):
    seq, table = np.array([9, -3, 2**31 - 1], dtype=np.int32), np.arange(12, dtype=np.int32).reshape(3, 4)
    free, done = np.full(5, -1, dtype=np.int32), np.array([1, 2, 255], dtype=np.uint8)
    want = ref.release(done, seq, table, free, 1, 4)
    got = cuda(free)
    seq_out, count_out = ops.pages_release(cuda(done), cuda(seq), cuda(table), got, cuda(np.array([1], dtype=np.int32)), 4)
    assert np.array_equal(got.cpu().numpy(), want["free_pages"]) and int(count_out) == 5 and not seq_out.any()


# ----------------------------------------------------------------------------------------------------------------------
# rotary positions
# ----------------------------------------------------------------------------------------------------------------------
def rope_case(ops, dim, rotary, n_axes, pairs, scale=1.0):
    half = rotary // 2
    axes = [(i * n_axes) // max(half, 1) for i in range(half)]
    freq = [10000.0 ** (-2.0 * i / rotary) for i in range(half)]
    return ops.RopePlan(dim, rotary, inv_freq=freq, axes=axes, pairs=pairs, scale=scale), freq, axes


def check_rotated(got, x, pos, freq, axes, pairs, dtype, scale=1.0, inverse=False):
    x = f64(x)
    want = ref.rotate(x, pos, freq, axes, pairs, scale, inverse)
    bound = ref.rotate_bound(x, len(freq), pairs, dtype, want, scale)
    off = np.abs(f64(got) - want)
    assert (off <= bound).all(), (off - bound).max()


@pytest.mark.parametrize("pairs", ["half", "adjacent"])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("dim,rotary", [(128, 128), (64, 64), (80, 40), (96, 32), (256, 256), (6, 4), (7, 2), (64, 0), (130, 130), (256, 64)])
def test_rotate(ops, dim, rotary, dtype, pairs):
    torch.manual_seed(dim + rotary)
    n_axes = 3 if rotary >= 6 else 1
    plan, freq, axes = rope_case(ops, dim, rotary, n_axes, pairs)
    for tokens, heads in ((1, 1), (5, 3), (67, 9)):
        pos = np.random.default_rng(tokens).integers(0, 40000, (n_axes, tokens))
        q = torch.randn(tokens, heads, dim, device="cuda", dtype=TYPES[dtype])
        k = torch.randn(tokens, 2, dim, device="cuda", dtype=TYPES[dtype])
        q_before = q.clone()
        a, b = plan.rotate([q, k], cuda(pos.astype(np.int32)))
        assert torch.equal(q, q_before)
        check_rotated(a, q, pos, freq, axes, pairs, dtype)
        check_rotated(b, k, pos, freq, axes, pairs, dtype)
        (c,) = plan.rotate([q], cuda(pos.astype(np.int64)), inverse=True)
        check_rotated(c, q, pos, freq, axes, pairs, dtype, inverse=True)


@pytest.mark.parametrize("offset", [0, 1, 2, 4, 8])
def test_rotate_takes_strided_views_and_misaligned_ones(ops, offset):
    """views of a fused projection, heads before tokens, shared (stride 0) heads, and starts off the vector grid"""
    plan, freq, axes = rope_case(ops, 64, 64, 1, "half")
    tokens, heads = 19, 5
    pos = np.arange(100, 100 + tokens)[None]
    flat = torch.randn(tokens * (3 * heads * 64 + 8) + 64, device="cuda", dtype=torch.bfloat16)
    fused = flat[offset : offset + tokens * 3 * heads * 64].view(tokens, 3 * heads, 64)
    by_head = torch.randn(heads, tokens, 64, device="cuda", dtype=torch.bfloat16).transpose(0, 1)
    shared = torch.randn(tokens, 1, 64, device="cuda", dtype=torch.bfloat16).expand(tokens, heads, 64)
    xs = [fused[:, :heads], fused[:, heads : 2 * heads], by_head, shared]
    for x, y in zip(xs, plan.rotate(xs, cuda(pos.astype(np.int32))[0])):
        check_rotated(y, x, pos, freq, axes, "half", "bf16")


def test_rotate_in_place_inside_a_fused_projection(ops):
    plan, freq, axes = rope_case(ops, 128, 64, 1, "half")
    fused = torch.randn(33, 12, 128, device="cuda", dtype=torch.float16)
    before = fused.clone()
    q, k = fused[:, :8], fused[:, 8:10]
    pos = np.arange(33)[None]
    plan.rotate([q, k], cuda(pos[0].astype(np.int32)), outs=[q, k])
    check_rotated(q, before[:, :8], pos, freq, axes, "half", "fp16")
    check_rotated(k, before[:, 8:10], pos, freq, axes, "half", "fp16")
    assert torch.equal(fused[:, 10:], before[:, 10:]) and torch.equal(fused[:, :10, 64:], before[:, :10, 64:])


def test_rotate_is_exact_at_far_and_negative_positions(ops):
    plan, freq, axes = rope_case(ops, 64, 64, 1, "half")
    pos = np.array([[0, 1, -1, -4097, 2**20 + 1, 2**31 - 1, -(2**31), 2**40 + 12345, -(2**45) - 7]])
    x = torch.randn(pos.shape[1], 3, 64, device="cuda")
    # beyond 2^31 the phase's own rounding (2^-65 turns a position) counts: 2^45 * 2^-65 * 2 pi < 2^-17
    got = plan.rotate([x], cuda(pos[0]))[0]
    x64 = f64(x)
    want = ref.rotate(x64, pos, freq, axes, "half")
    bound = ref.rotate_bound(x64, 32, "half", "fp32", want)
    far = np.abs(pos[0]).astype(float)[:, None, None] * 2.0**-65 * 2 * math.pi * (np.abs(x64).max() * 2)
    # the reference takes inv_freq's double as it is; so does the plan, up to its 64-bit fraction
    assert (np.abs(f64(got) - want) <= bound + far).all()


def test_rotate_scale_and_many_rows(ops):
    plan, freq, axes = rope_case(ops, 128, 128, 2, "adjacent", scale=1.37)
    tokens = 3001
    pos = np.stack([np.arange(tokens), np.arange(tokens)[::-1]])
    x = torch.randn(tokens, 7, 128, device="cuda", dtype=torch.bfloat16)
    (y,) = plan.rotate([x], cuda(pos.astype(np.int32)))
    check_rotated(y, x, pos, freq, axes, "adjacent", "bf16", scale=1.37)


def test_rotate_of_no_tokens(ops):
    plan, _, _ = rope_case(ops, 64, 64, 1, "half")
    (y,) = plan.rotate([torch.empty(0, 4, 64, device="cuda")], torch.empty(0, dtype=torch.int32, device="cuda"))
    assert y.shape == (0, 4, 64)


@pytest.mark.parametrize("pairs", ["half", "adjacent"])
def test_rotate_gradient(ops, pairs):
    """Against the formula (the transposed turn), against differences, and through shared heads."""
    plan, freq, axes = rope_case(ops, 96, 64, 3, pairs, scale=0.8)
    pos = np.random.default_rng(3).integers(0, 3000, (3, 41))
    p = cuda(pos.astype(np.int32))
    q = torch.randn(41, 6, 96, device="cuda", requires_grad=True)
    k1 = torch.randn(41, 1, 96, device="cuda", requires_grad=True)
    gq, gk = torch.randn(41, 6, 96, device="cuda"), torch.randn(41, 4, 96, device="cuda")
    a, b = plan.rotate([q, k1.expand(41, 4, 96)], p)
    ga, gb = torch.autograd.grad([a, b], [q, k1], [gq, gk])
    check_rotated(ga, gq, pos, freq, axes, pairs, "fp32", scale=0.8, inverse=True)
    want = ref.rotate(f64(gk), pos, freq, axes, pairs, 0.8, True).sum(1, keepdims=True)
    # four rows, each within 16 units of 2^-24 of its pair's size (at most twice the largest value), and their sum
    assert np.abs(f64(gb) - want).max() <= 4 * 40 * 2.0**-24 * np.abs(f64(gk)).max()
    # the operator is linear: a central difference along d is exact up to rounding, 2^-24 of the values' size each way
    d = torch.randn_like(q)
    with torch.no_grad():
        up, down = plan.rotate([q + d, q - d], p)
    diff = float(((up.double() - down.double()) / 2 * gq.double()).sum())
    dot = float((ga.double() * d.double()).sum())
    assert abs(diff - dot) <= 40 * 2.0**-24 * float((gq.abs() * (q.detach().abs() + d.abs()).max()).sum())
    # a gradient that is one number repeated (stride 0) and a second backward
    (one,) = torch.autograd.grad(plan.rotate([q], p)[0].sum(), [q])
    check_rotated(one, torch.ones(41, 6, 96), pos, freq, axes, pairs, "fp32", scale=0.8, inverse=True)


# ----------------------------------------------------------------------------------------------------------------------
# append
# ----------------------------------------------------------------------------------------------------------------------
def make_cache(pages, page, heads, dim, dtype, layout, extra=0):
    """A cache whose every byte is set, in either order of memory, with `extra` elements between heads."""
    shape = (pages, page, heads, dim + extra) if layout == "token" else (pages, heads, page, dim + extra)
    x = torch.randn(shape, device="cuda").to(TYPES[dtype])
    return (x if layout == "token" else x.transpose(1, 2))[..., :dim]


@pytest.mark.parametrize("layout", ["token", "head"])
@pytest.mark.parametrize("dtype,cache_dtype", [("bf16", "bf16"), ("fp16", "fp16"), ("bf16", "e4m3"), ("fp16", "e4m3")])
@pytest.mark.parametrize("tokens,q_heads,heads,dim,rotary,page", [(1, 1, 1, 64, 64, 1), (37, 8, 2, 128, 128, 16), (130, 6, 3, 80, 40, 5), (9, 2, 2, 6, 4, 3)])
def test_append(ops, tokens, q_heads, heads, dim, rotary, page, dtype, cache_dtype, layout):
    torch.manual_seed(tokens)
    r = np.random.default_rng(tokens)
    n_axes = 3 if rotary >= 6 else 1
    plan, freq, axes = rope_case(ops, dim, rotary, n_axes, "half")
    pages = tokens // page + 3
    scale = (0.031, 1.7) if cache_dtype == "e4m3" else (1.0, 1.0)
    k, v = make_cache(pages, page, heads, dim, cache_dtype, layout, 16), make_cache(pages, page, heads, dim, cache_dtype, layout)
    k0, v0 = f64(k), f64(v)
    fused = torch.randn(tokens, (q_heads + 2 * heads) * dim, device="cuda", dtype=TYPES[dtype])
    q, kk, vv = (x.unflatten(1, (-1, dim)) for x in fused.split([q_heads * dim, heads * dim, heads * dim], 1))
    pos = r.integers(0, 9000, (n_axes, tokens))
    slots = r.permutation(pages * page)[:tokens].astype(np.int32)
    if tokens > 5:
        slots[[1, 3, 4]] = [-1, pages * page, 2**31 - 1]  # none, and two that are not there
    cache = ops.PagedCache(k, v, k_scale=scale[0], v_scale=scale[1])
    out = plan.append(q, kk, vv, cuda(pos.astype(np.int32)), cuda(slots), cache)
    check_rotated(out, q, pos, freq, axes, "half", dtype)
    kept = (slots >= 0) & (slots < pages * page)
    for got, before, x, s, turned in ((k, k0, kk, scale[0], True), (v, v0, vv, scale[1], False)):
        x = f64(x)
        y = ref.rotate(x, pos, freq, axes, "half") if turned else x
        bound = ref.rotate_bound(x, len(freq), "half", cache_dtype, y) / s
        y = y / s
        if cache_dtype == "e4m3":
            y = np.clip(y, -448, 448)
            bound += 2.0**-10 + 2.0**-22 * np.abs(y)  # half the smallest step; the division by the scale
        want, allowed = before.reshape(-1, heads, dim).copy(), np.zeros((pages * page, heads, dim))
        want[slots[kept]], allowed[slots[kept]] = y[kept], bound[kept]
        assert (np.abs(f64(got).reshape(-1, heads, dim) - want) <= allowed).all()


def test_append_keeps_nan_and_clamps_infinity_in_8_bits(ops):
    plan, _, _ = rope_case(ops, 16, 0, 1, "half")
    k, v = make_cache(1, 4, 1, 16, "e4m3", "token"), make_cache(1, 4, 1, 16, "e4m3", "token")
    x = torch.zeros(2, 1, 16, device="cuda", dtype=torch.bfloat16)
    x[0, 0, :4] = torch.tensor([math.nan, math.inf, -math.inf, 1e30])
    plan.append(x, x, x, torch.zeros(2, dtype=torch.int32, device="cuda"), torch.tensor([2, 0], dtype=torch.int32, device="cuda"), ops.PagedCache(k, v))
    got = f64(v)[0, 2, 0]
    assert np.isnan(got[0]) and got[1] == 448 and got[2] == -448 and got[3] == 448 and not got[4:].any()
    assert not f64(v)[0, 0].any()


# ----------------------------------------------------------------------------------------------------------------------
# attention
# ----------------------------------------------------------------------------------------------------------------------
def attend_inputs(r, lens, q_heads, heads, dim, page, dtype, cache_dtype, layout, poison=True, extra=0):
    lens = np.asarray(lens, dtype=np.int32)
    n, have = len(lens), -(-np.maximum(lens, 0) // page)
    row = max(1, int(have.max()))
    pages = int(have.sum()) + 2
    numbers = r.permutation(pages).astype(np.int32)
    table = np.full((n, row), -1, dtype=np.int32)
    live = np.zeros((pages, page), dtype=bool)
    at = 0
    for i in range(n):
        table[i, : have[i]] = numbers[at : at + have[i]]
        for j in range(have[i]):
            live[table[i, j], : min(page, lens[i] - j * page)] = True
        at += have[i]
    k, v = make_cache(pages, page, heads, dim, cache_dtype, layout, extra), make_cache(pages, page, heads, dim, cache_dtype, layout, extra)
    if poison:  # what no request holds may be anything
        dead = torch.from_numpy(~live).cuda()[..., None, None].expand(k.shape)
        if cache_dtype == "e4m3":
            k.copy_(torch.where(dead, torch.full_like(k.float(), math.nan), k.float()).to(k.dtype))
            v.copy_(torch.where(dead, torch.full_like(v.float(), math.nan), v.float()).to(v.dtype))
        else:
            k.masked_fill_(dead, math.nan)
            v.masked_fill_(dead, math.inf)
    q = torch.randn(n, q_heads, dim, device="cuda", dtype=TYPES[dtype]) * 2
    return q, k, v, table, lens


def check_attend(ops, q, k, v, table, lens, page, dtype, scales=(1.0, 1.0), window=0, softcap=0.0, plan=None, scale=None):
    n, q_heads, dim = q.shape
    plan = plan or ops.AttendPlan(n, q_heads, k.shape[2], dim, window=window, softcap=softcap, scale=scale)
    cache = ops.PagedCache(k, v, k_scale=scales[0], v_scale=scales[1])
    out, lse = plan.attend(q, cache, cuda(table), cuda(lens), return_lse=True)
    k64, v64 = f64(k) * scales[0], f64(v) * scales[1]
    with np.errstate(invalid="ignore"):
        want, want_lse, size, mass = ref.attend(f64(q), k64, v64, table, lens, plan.scale, window, softcap)
    bound, lse_bound = ref.attend_bound(want, size, mass, dim, dtype)
    got, got_lse = f64(out), f64(lse)
    assert np.isfinite(got).all()
    assert (np.abs(got - want) <= bound).all(), (np.abs(got - want) / bound).max()
    there = np.isfinite(want_lse)
    assert np.array_equal(there, np.isfinite(got_lse)) and (got_lse[~there] == -np.inf).all()
    assert (np.abs(got_lse[there] - want_lse[there]) <= lse_bound[there] + 2.0**-22 * np.abs(want_lse[there])).all()
    again, _ = plan.attend(q, cache, cuda(table), cuda(lens), return_lse=True)
    assert torch.equal(out, again)  # the parts are joined in a fixed order
    return out


LENS = [1, 0, 17, 64, 65, 130, 2, 63, 1000, 128]


@pytest.mark.parametrize("dtype,cache_dtype", [("bf16", "bf16"), ("fp16", "fp16"), ("bf16", "e4m3"), ("fp16", "e4m3")])
@pytest.mark.parametrize("dim", [16, 64, 80, 128, 160, 256])
@pytest.mark.parametrize("q_heads,heads", [(1, 1), (8, 2), (32, 4), (14, 2), (16, 1), (24, 1)])
def test_attend(ops, q_heads, heads, dim, dtype, cache_dtype):
    r = np.random.default_rng(dim + q_heads)
    torch.manual_seed(dim + q_heads)
    scales = (0.7, 1.3) if cache_dtype == "e4m3" else (1.0, 1.0)
    layout = "head" if dim % 64 else "token"
    q, k, v, table, lens = attend_inputs(r, LENS, q_heads, heads, dim, 16, dtype, cache_dtype, layout)
    check_attend(ops, q, k, v, table, lens, 16, dtype, scales)


@pytest.mark.parametrize("layout", ["token", "head"])
@pytest.mark.parametrize("page", [1, 3, 8, 24, 48, 64, 256])
def test_attend_pages_that_end_inside_a_tile(ops, page, layout):
    r = np.random.default_rng(page)
    torch.manual_seed(page)
    q, k, v, table, lens = attend_inputs(r, LENS, 8, 2, 128, page, "bf16", "bf16", layout, extra=8)
    check_attend(ops, q, k, v, table, lens, page, "bf16")


@pytest.mark.parametrize("window", [1, 2, 63, 64, 65, 400, 100000])
@pytest.mark.parametrize("softcap", [0.0, 5.0])
def test_attend_window_and_softcap(ops, window, softcap):
    r = np.random.default_rng(window)
    torch.manual_seed(window)
    q, k, v, table, lens = attend_inputs(r, LENS, 6, 2, 64, 16, "fp16", "fp16", "token")
    check_attend(ops, q, k, v, table, lens, 16, "fp16", window=window, softcap=softcap)


@pytest.mark.parametrize("requests", [1, 3, 40, 700])
def test_attend_many_requests(ops, requests):
    r = np.random.default_rng(requests)
    torch.manual_seed(requests)
    lens = r.integers(0, 300, requests)
    lens[0] = 7000 if requests < 100 else 300
    q, k, v, table, lens = attend_inputs(r, lens, 4, 2, 64, 16, "bf16", "bf16", "token")
    check_attend(ops, q, k, v, table, lens, 16, "bf16")


@pytest.mark.parametrize("q_heads,heads", [(1, 1), (16, 1), (64, 1), (40, 8)])
def test_attend_one_long_request(ops, q_heads, heads):
    r = np.random.default_rng(q_heads)
    torch.manual_seed(q_heads)
    q, k, v, table, lens = attend_inputs(r, [30011], q_heads, heads, 128, 32, "bf16", "bf16", "head")
    check_attend(ops, q, k, v, table, lens, 32, "bf16")


@pytest.mark.parametrize("q_heads,heads", [(64, 64), (37, 37), (80, 40), (70, 35)])
@pytest.mark.parametrize("page", [3, 16])
def test_attend_more_heads_than_a_team_has_blocks(ops, q_heads, heads, page):
    """The heads of a request go round by round through the teams: with requests that end inside pieces, an empty one, and
    one that many pieces share."""
    r = np.random.default_rng(heads + page)
    torch.manual_seed(heads + page)
    q, k, v, table, lens = attend_inputs(r, [700, 0, 65, 3001, 1, 128], q_heads, heads, 64, page, "bf16", "bf16", "token")
    check_attend(ops, q, k, v, table, lens, page, "bf16")
    check_attend(ops, q, k, v, table, lens, page, "bf16", window=300)


def test_one_plan_serves_fewer_requests_and_other_caches(ops):
    """The workspace is left ready by every call, whatever the calls before it split."""
    r = np.random.default_rng(11)
    torch.manual_seed(11)
    plan = ops.AttendPlan(40, 8, 2, 128)
    for lens, cache_dtype, page in (([9000], "bf16", 16), ([5] * 40, "e4m3", 8), ([4000, 1, 0, 777], "bf16", 5), ([9000], "e4m3", 64), (list(range(0, 4000, 100)), "bf16", 16)):
        q, k, v, table, lens = attend_inputs(r, lens, 8, 2, 128, page, "bf16", cache_dtype, "token")
        check_attend(ops, q, k, v, table, lens, page, "bf16", plan=plan)
    assert not plan.failed()


def test_attend_of_empty_requests_only(ops):
    r = np.random.default_rng(0)
    q, k, v, table, lens = attend_inputs(r, [0, 0, -5], 8, 2, 64, 16, "bf16", "bf16", "token")
    out = check_attend(ops, q, k, v, table, lens, 16, "bf16")
    assert not out.any()


def test_attend_holes_and_lengths_beyond_the_table(ops):
    """Table entries that are no pages take no part (all of a request's, some, the last); a length beyond the row is cut."""
    r = np.random.default_rng(5)
    q, k, v, table, lens = attend_inputs(r, [200, 200, 200, 40], 8, 2, 64, 16, "bf16", "bf16", "token", poison=False)
    table[0, :] = -1
    table[1, [0, 3, 4, 5, 6, 7]] = [-1, 10**6, -(2**31), 2**31 - 1, -1, k.shape[0]]
    table[2, 12] = -1
    lens[3] = 2**31 - 1
    table[3, :] = table[2, ::-1]
    check_attend(ops, q, k, v, table, lens, 16, "bf16")


def test_attend_extreme_scores(ops):
    """Scores far apart (all weight on one token), equal ones, and zero queries."""
    r = np.random.default_rng(6)
    q, k, v, table, lens = attend_inputs(r, [500, 500, 500], 8, 2, 64, 16, "fp16", "fp16", "token")
    q[0] *= 500
    q[1] = 0
    check_attend(ops, q, k, v, table, lens, 16, "fp16")
    q, k, v, table, lens = attend_inputs(r, [500], 8, 2, 64, 16, "bf16", "bf16", "token")
    check_attend(ops, q * 1e4, k, v, table, lens, 16, "bf16")
    q, k, v, table, lens = attend_inputs(r, [500, 30], 8, 2, 64, 16, "bf16", "e4m3", "token")
    q[0] *= 1e30  # beyond fp16's range
    q[1] *= 1e-30
    check_attend(ops, q, k, v, table, lens, 16, "bf16", scales=(1e-30, 1.0), scale=0.125)


def test_attend_nan_and_infinity_of_live_tokens_come_through(ops):
    r = np.random.default_rng(7)
    q, k, v, table, lens = attend_inputs(r, [100, 100, 100], 4, 2, 64, 16, "bf16", "bf16", "token")
    k[table[0, 2], 3, 0, 5] = math.nan
    v[table[1, 2], 3, 1, 7] = math.inf
    plan = ops.AttendPlan(3, 4, 2, 64)
    out = f64(plan.attend(q, ops.PagedCache(k, v), cuda(table), cuda(lens)))
    assert np.isnan(out[0, :2]).all() and np.isfinite(out[0, 2:]).all()
    assert (out[1, 2:, 7] == np.inf).all() and np.isfinite(np.delete(out[1, 2:], 7, 1)).all() and np.isfinite(out[1, :2]).all()
    assert np.isfinite(out[2]).all()


def test_attend_cache_offsets_beyond_32_bits(ops):
    """Pages whose first element lies past 2^32 bytes: one tensor, three gigabytes apart, of which a few pages are used."""
    page, heads, dim = 16, 8, 128
    pages = 3 * 2**32 // (page * heads * dim * 2)
    k = torch.zeros(pages, page, heads, dim, device="cuda", dtype=torch.bfloat16)
    v = torch.zeros(pages, page, heads, dim, device="cuda", dtype=torch.bfloat16)
    used = np.array([[pages - 1, 3, pages // 2 + 1, pages - 7]], dtype=np.int32)
    for p in used[0]:
        k[p], v[p] = torch.randn_like(k[p]), torch.randn_like(v[p])
    q = torch.randn(1, 16, dim, device="cuda", dtype=torch.bfloat16)
    out = ops.AttendPlan(1, 16, heads, dim).attend(q, ops.PagedCache(k, v), cuda(used), cuda(np.array([61], dtype=np.int32)))
    few = torch.from_numpy(used[0].astype(np.int64)).cuda()
    want, _, size, mass = ref.attend(f64(q), f64(k[few]), f64(v[few]), np.array([[0, 1, 2, 3]]), [61], dim**-0.5)
    bound, _ = ref.attend_bound(want, size, mass, dim, "bf16")
    assert (np.abs(f64(out) - want) <= bound).all()
    # and the write of a token there
    plan, freq, axes = rope_case(ops, dim, dim, 1, "half")
    x = torch.randn(1, heads, dim, device="cuda", dtype=torch.bfloat16)
    plan.append(x, x, x, cuda(np.array([5], dtype=np.int32)), cuda(np.array([(pages - 2) * page + 9], dtype=np.int32)), ops.PagedCache(k, v))
    assert torch.equal(v[pages - 2, 9], x[0])


def test_attend_strided_q_and_output(ops):
    r = np.random.default_rng(8)
    q, k, v, table, lens = attend_inputs(r, [100, 3], 8, 2, 64, 16, "bf16", "bf16", "token")
    want = ops.AttendPlan(2, 8, 2, 64).attend(q, ops.PagedCache(k, v), cuda(table), cuda(lens))
    odd = torch.zeros(2 * 8 * 67 + 3, device="cuda", dtype=torch.bfloat16)[3:].view(2, 8, 67)
    odd[..., :64] = q
    held = torch.zeros(8, 2, 65, device="cuda", dtype=torch.bfloat16)
    out = held.transpose(0, 1)[..., 1:]
    wide = cuda(np.pad(table, ((0, 0), (0, 5)), constant_values=10**6))[:, : table.shape[1]]
    ops.AttendPlan(2, 8, 2, 64).attend(odd[..., :64], ops.PagedCache(k, v), wide, cuda(lens), out=out)
    assert torch.equal(out, want) and not held[..., 0].any()


# ----------------------------------------------------------------------------------------------------------------------
# streams, graphs, a step from end to end
# ----------------------------------------------------------------------------------------------------------------------
def test_calls_on_other_streams(ops):
    r = np.random.default_rng(9)
    q, k, v, table, lens = attend_inputs(r, [3000, 100], 8, 2, 128, 16, "bf16", "bf16", "token")
    plan, cache = ops.AttendPlan(2, 8, 2, 128), ops.PagedCache(k, v)
    t, n = cuda(table), cuda(lens)
    want = plan.attend(q, cache, t, n)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    got = [plan.attend(q, cache, t, n, stream=streams[i % 3]) for i in range(12)]  # one workspace, three streams
    torch.cuda.synchronize()
    assert all(torch.equal(g, want) for g in got)
    rope, _, _ = rope_case(ops, 128, 128, 1, "half")
    pos = torch.tensor([4, 5], dtype=torch.int32, device="cuda")
    want = rope.rotate([q], pos)[0]
    torch.cuda.synchronize()
    got = rope.rotate([q], pos, stream=streams[0])[0]
    streams[0].synchronize()
    assert torch.equal(got, want)


def test_a_decoding_step_in_a_graph(ops):
    """pages, append and attention captured once and replayed for several steps, against the definitions."""
    torch.manual_seed(1)
    n, q_heads, heads, dim, page, row = 5, 8, 2, 64, 4, 8
    pages = n * row
    table = torch.full((n, row), -1, dtype=torch.int32, device="cuda")
    free = torch.randperm(pages, device="cuda").to(torch.int32)
    seq, count = torch.zeros(n, dtype=torch.int32, device="cuda"), torch.tensor([pages], dtype=torch.int32, device="cuda")
    new = torch.tensor([1, 0, 1, 1, 1], dtype=torch.int32, device="cuda")
    k = torch.zeros(pages, page, heads, dim, device="cuda", dtype=torch.float16)
    v = torch.zeros_like(k)
    cache, attention = ops.PagedCache(k, v), ops.AttendPlan(n, q_heads, heads, dim)
    rope, freq, axes = rope_case(ops, dim, dim, 1, "half")
    fused = torch.zeros(n, q_heads + 2 * heads, dim, device="cuda", dtype=torch.float16)

    def step():
        s = ops.pages_extend(new, seq, table, free, count, page, n)
        q = rope.append(fused[:, :q_heads], fused[:, q_heads : q_heads + heads], fused[:, q_heads + heads :], s.positions, s.slots, cache)
        rows = torch.zeros(n + 1, q_heads, dim, device="cuda", dtype=q.dtype)  # the last takes what is no request's
        rows[torch.where(s.requests < 0, n, s.requests).long()] = q
        out = attention.attend(rows[:n], cache, table, s.seq_lens)
        seq.copy_(s.seq_lens)
        count.copy_(s.free_count)
        return q, out, s

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    seq.zero_()
    count.fill_(pages)
    table.fill_(-1)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        q, out, s = step()
    ks = [[] for _ in range(n)]
    vs = [[] for _ in range(n)]
    live = [0, 2, 3, 4]
    for t in range(11):
        fused.normal_()
        graph.replay()
        torch.cuda.synchronize()
        x = f64(fused)
        assert s.requests.tolist() == live + [-1] and seq.tolist() == [t + 1, 0, t + 1, t + 1, t + 1]
        for i, r in enumerate(live):
            turned = ref.rotate(x[i : i + 1, q_heads : q_heads + heads], np.array([[t]]), freq, axes, "half")[0]
            ks[r].append(turned.astype(np.float16).astype(float))
            vs[r].append(x[i, q_heads + heads :])
            q_want = ref.rotate(x[i : i + 1, :q_heads], np.array([[t]]), freq, axes, "half")
            want, _, size, mass = ref.attend(f64(q)[i : i + 1], np.array(ks[r])[:, None], np.array(vs[r])[:, None],
                                             np.arange(t + 1)[None], [t + 1], dim**-0.5)
            bound, _ = ref.attend_bound(want, size, mass, dim, "fp16")
            assert np.abs(f64(q)[i] - q_want[0]).max() <= 2.0**-10 * 8
            # k may be rounded to the other neighbour: 2^-11 of each product, on top
            assert (np.abs(f64(out)[r] - want[0]) <= bound[0] + 2 * 2.0**-10 * (size[0, :, None] * mass[0])).all()
        assert not out[1].any()


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_the_example_runs(cache):
    import os
    import subprocess
    import sys

    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    said = subprocess.run([sys.executable, os.path.join(root, "examples", "decode_step.py"), "--cache", cache, "--steps", "5"],
                          capture_output=True, text=True, timeout=300)
    assert said.returncode == 0, said.stderr[-2000:]
    assert "5 decoding steps" in said.stdout
