"""The cache of 4 bits on the GPU, written, read back and attended to, against the definitions in 64 bits."""
import numpy as np
import pytest

import packed_ref as ref
import serve_ref

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SHAPES = [(64, 32), (64, 64), (96, 32), (128, 32), (128, 64), (256, 32), (256, 64)]


@pytest.fixture(scope="module")
def ops():
    from paper_2002_12798_b200 import ops

    return ops


def f64(t):
    return t.to(torch.float32).cpu().double().numpy()


def cuda(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(dtype)


def check_read(ops, cache, slots, k, v, group):
    """The cache holds what the definition makes of k and v (float64 [tokens, heads, dim]) at the slots, bit for bit."""
    for name in ("fp32", "bf16", "fp16"):
        got = cache.read(slots, dtype=TYPES[name])
        for x, y in zip((k, v), got):
            want = torch.from_numpy(ref.values(*ref.quantise(x, group))).to(torch.float32).to(TYPES[name])
            assert y.dtype == TYPES[name] and np.array_equal(f64(y), f64(want), equal_nan=True), name


# ----------------------------------------------------------------------------------------------------------------------
# written and read back
# ----------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dim,group", SHAPES)
@pytest.mark.parametrize("tokens,heads,page", [(1, 1, 16), (37, 3, 48), (200, 8, 32)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_write_and_read(ops, dim, group, tokens, heads, page, dtype):
    r = np.random.default_rng(dim + group + tokens)
    pages = tokens // page + 3
    x = r.standard_normal((2, tokens, heads, dim)) * np.exp(r.standard_normal((2, tokens, heads, 1)) * 2)
    x[0] += r.standard_normal(dim) * 4
    k, v = (cuda(y, TYPES[dtype]) for y in x)
    slots = cuda(r.permutation(pages * page)[:tokens].astype(np.int32))
    cache = ops.PackedCache.zeros(pages, page, heads, dim, group=group)
    cache.data.fill_(255)
    before = cache.data.clone()
    assert cache.write(k, v, slots) is None
    check_read(ops, cache, slots, f64(k), f64(v), group)
    # every other token's bytes are as they were
    other = torch.ones(pages * page, dtype=torch.bool, device="cuda")
    other[slots.long()] = False
    rest = other.nonzero()[:, 0].to(torch.int32)
    fresh = ops.PackedCache(before, page, dim, group=group)
    for a, b in zip(cache.read(rest, dtype=torch.float32), fresh.read(rest, dtype=torch.float32)):
        assert torch.equal(a.view(torch.int32), b.view(torch.int32))
    assert int((cache.data != before).sum()) <= tokens * heads * (dim + 8 * dim // group)


@pytest.mark.parametrize("scale", [1e-38, 3e-5, 1.0, 1e4, 1e37])
def test_groups_of_every_size(ops, scale):
    """Values near both ends of bf16, equal ones, ones on the border between two codes, zeros of both signs."""
    r = np.random.default_rng(3)
    x = r.standard_normal((64, 2, 128)) * scale
    x[1] = 0.0
    x[2] = -0.0
    x[3, :, ::2] = -0.0
    x[4] = scale
    x[5] = np.arange(128) % 31 * scale / 4  # every second one lies on a border
    x[6, :, 5] = 30 * scale  # an outlier
    x[7, 0] = r.integers(-3, 4, 128) * 2.0**-133
    x[8] = -scale * 2.0 ** -(np.arange(128) % 60.0)
    k = cuda(x, torch.bfloat16)
    for group in (32, 64):
        cache = ops.PackedCache.zeros(4, 16, 2, 128, group=group)
        slots = torch.arange(64, device="cuda", dtype=torch.int32)
        cache.write(k, k.flip(0).contiguous(), slots)
        check_read(ops, cache, slots, f64(k), f64(k)[::-1], group)


def test_groups_without_finite_numbers(ops):
    x = torch.randn(16, 2, 128, device="cuda", dtype=torch.bfloat16)
    x[0, 0, 3] = float("nan")
    x[1, 1, 70] = float("inf")
    x[2, 0, 127] = -float("inf")
    x[3] = float("nan")
    cache = ops.PackedCache.zeros(1, 16, 2, 128, group=32)
    slots = torch.arange(16, device="cuda", dtype=torch.int32)
    cache.write(x, x, slots)
    check_read(ops, cache, slots, f64(x), f64(x), 32)
    k = cache.read(slots)[0]
    assert k[0, 0, :32].isnan().all() and not k[0, 0, 32:].isnan().any() and k[3].isnan().all() and not k[4:].isnan().any()


def test_slots_that_there_are_not(ops):
    x = torch.randn(6, 2, 64, device="cuda", dtype=torch.float16)
    cache = ops.PackedCache.zeros(2, 16, 2, 64)
    slots = torch.tensor([3, -1, 31, 32, 2**31 - 1, -(2**31)], device="cuda", dtype=torch.int32)
    cache.write(x, x, slots)
    k, v = cache.read(slots)
    assert not k[[1, 3, 4, 5]].any() and not v[[1, 3, 4, 5]].any()
    whole = cache.read(torch.arange(32, device="cuda", dtype=torch.int32))[0]
    assert set(whole.any(-1).any(-1).nonzero()[:, 0].tolist()) == {3, 31}
    none = torch.empty(0, device="cuda", dtype=torch.int32)
    assert cache.read(none)[0].shape == (0, 2, 64) and cache.write(x[:0], x[:0], none) is None


@pytest.mark.parametrize("pairs", ["half", "adjacent"])
@pytest.mark.parametrize("dim,rotary,group,q_heads,kv_heads,dtype", [
    (128, 128, 64, 32, 8, "bf16"), (128, 128, 32, 7, 1, "fp16"), (64, 64, 64, 4, 2, "bf16"), (96, 96, 32, 6, 6, "bf16"), (256, 256, 64, 3, 3, "fp16"),
    (128, 64, 32, 8, 2, "bf16"), (128, 40, 64, 8, 2, "fp16"), (96, 2, 32, 4, 2, "bf16"), (64, 0, 32, 2, 1, "bf16"), (256, 200, 32, 2, 40, "bf16"),
])
def test_append(ops, dim, rotary, group, q_heads, kv_heads, dtype, pairs):
    r = np.random.default_rng(dim + rotary + q_heads)
    tokens, page, axes = 45, 16, 3
    half = rotary // 2
    freq = [10000.0 ** (-2.0 * i / max(rotary, 1)) for i in range(half)]
    axis = [int(a) for a in r.integers(0, axes, half)]
    if half:
        axis[0] = axes - 1
    x = cuda(r.standard_normal((tokens, q_heads + 2 * kv_heads, dim)), TYPES[dtype])
    q, k, v = x[:, :q_heads], x[:, q_heads : q_heads + kv_heads], x[:, q_heads + kv_heads :]
    positions = r.integers(0, 100_000, (axes, tokens)).astype(np.int64)
    positions[:, 0] = [0, 2**31 - 1, -5]
    slots = r.permutation(4 * page)[:tokens].astype(np.int32)
    slots[7] = -1
    rope = ops.RopePlan(dim, rotary, inv_freq=freq, axes=axis, pairs=pairs, scale=1.25)
    cache = ops.PackedCache.zeros(4, page, kv_heads, dim, group=group)
    wide = positions.astype(np.int64) if dim == 128 else positions.astype(np.int32)
    out = rope.append(q, k, v, cuda(wide), cuda(slots), cache)
    same = rope.rotate([q.contiguous()], cuda(wide))[0]
    assert torch.equal(out, same)  # q as every other cache has it
    live = slots >= 0
    turned = serve_ref.rotate(f64(k), positions, freq, axis, pairs, scale=1.25)
    check_read(ops, cache, cuda(slots[live]), turned[live], f64(v)[live], group)


@pytest.mark.parametrize("offset,row_pad", [(0, 0), (1, 0), (3, 5), (8, 8)])
def test_append_from_rows_of_any_alignment(ops, offset, row_pad):
    r = np.random.default_rng(offset)
    tokens, q_heads, heads, dim = 33, 4, 2, 128
    width = (q_heads + 2 * heads) * dim
    flat = torch.randn(offset + tokens * (width + row_pad), device="cuda", dtype=torch.bfloat16)
    x = flat[offset:].as_strided((tokens, q_heads + 2 * heads, dim), (width + row_pad, dim, 1), flat.storage_offset() + offset)
    q, k, v = x[:, :q_heads], x[:, q_heads : q_heads + heads], x[:, q_heads + heads :]
    slots = cuda(r.permutation(48)[:tokens].astype(np.int32))
    positions = torch.arange(tokens, device="cuda", dtype=torch.int32)
    cache = ops.PackedCache.zeros(3, 16, heads, dim)
    rope = ops.RopePlan(dim)
    want_k, want_v = f64(k), f64(v)
    out = rope.append(q, k, v, positions, slots, cache, out=q)  # in place
    freq = [10000.0 ** (-2.0 * i / dim) for i in range(dim // 2)]
    check_read(ops, cache, slots, serve_ref.rotate(want_k, positions.cpu().numpy()[None], freq, [0] * 64, "half"), want_v, 64)
    assert out.data_ptr() == q.data_ptr()


def test_read_into_views(ops):
    cache = ops.PackedCache.zeros(2, 32, 2, 96, group=32)
    x = torch.randn(64, 2, 96, device="cuda", dtype=torch.bfloat16)
    slots = torch.randperm(64, device="cuda").to(torch.int32)
    cache.write(x, -x, slots)
    plain = cache.read(slots)
    for pad in (0, 1, 8):  # one tensor for both, rows of every alignment
        both = torch.full((64, 2, 2, 96 + pad), 7.0, device="cuda", dtype=torch.bfloat16)
        views = both[:, 0, :, pad:], both[:, 1, :, pad:]
        got = cache.read(slots, out=views)
        assert torch.equal(views[0], plain[0]) and torch.equal(views[1], plain[1]) and got[0].data_ptr() == views[0].data_ptr()
        assert (both[..., :pad] == 7).all()


def test_memory_of_any_order(ops):
    """Heads outside pages, rows with room behind them, a part of a larger pool."""
    size = ops.PackedCache.page_bytes(32, 128, 32)
    pool = torch.full((3, 7, 2 * size + 32), 255, device="cuda", dtype=torch.uint8)
    x = torch.randn(100, 3, 128, device="cuda", dtype=torch.float16)
    slots = torch.randperm(5 * 32, device="cuda")[:100].to(torch.int32)
    view = pool[:, 1:6, 16 : 16 + size].transpose(0, 1)  # [pages, heads, bytes]
    cache = ops.PackedCache(view, 32, 128, group=32)
    cache.write(x, 2 * x, slots)
    check_read(ops, cache, slots, f64(x), 2 * f64(x), 32)
    assert (pool[:, 0] == 255).all() and (pool[:, 6] == 255).all() and (pool[..., :16] == 255).all() and (pool[..., 16 + size :] == 255).all()


# ----------------------------------------------------------------------------------------------------------------------
# attention
# ----------------------------------------------------------------------------------------------------------------------
def filled(ops, r, slots, page, heads, dim, group, dtype, k=None, v=None, fill=255):
    """A cache whose slots are all written, and what it holds; memory that is not written is set to `fill` before."""
    k = r.standard_normal((slots, heads, dim)) + 2 * r.standard_normal((heads, dim)) if k is None else k
    v = r.standard_normal((slots, heads, dim)) * np.exp(r.standard_normal((slots, 1, 1))) if v is None else v
    cache = ops.PackedCache.zeros(slots // page, page, heads, dim, group=group)
    cache.data.fill_(fill)
    kt, vt = cuda(k, TYPES[dtype]), cuda(v, TYPES[dtype])
    cache.write(kt, vt, torch.arange(slots, device="cuda", dtype=torch.int32))
    return cache, ref.quantise(f64(kt), group), ref.quantise(f64(vt), group)


def check_attend(plan, q, cache, table, lens, k, v, some=None):
    out, lse = plan.attend(q, cache, cuda(table), cuda(lens), return_lse=True)
    page, pages = cache.page_size, cache.pages
    got, got_lse, x = f64(out), lse.cpu().double().numpy(), f64(q)
    unit = serve_ref.UNIT["bf16" if q.dtype == torch.bfloat16 else "fp16"]
    for i in range(len(lens)) if some is None else some:
        n = min(max(int(lens[i]), 0), table.shape[1] * page)
        t = np.arange(max(0, n - plan.window) if plan.window else 0, n)
        number = table[i, t // page]
        at = (number * page + t % page)[(number >= 0) & (number < pages)]
        want, want_lse, bound, lse_bound = ref.attend(x[i], k, v, at, plan.scale, plan.softcap)
        tiny = 0 if unit == 2.0**-8 else 2.0**-25  # half of fp16's smallest step
        assert (np.abs(got[i] - want) <= bound + unit * (np.abs(want) + bound) + tiny).all(), (i, n)
        assert np.array_equal(np.isneginf(got_lse[i]), np.isneginf(want_lse)), (i, n)
        fine = ~np.isneginf(want_lse)
        assert (np.abs(got_lse[i] - want_lse)[fine] <= lse_bound[fine]).all(), (i, n)
    assert not plan.failed()
    return out, lse


LENGTHS = [0, 1, 15, 16, 17, 33, 127, 128, 129, 255, 300, 5]


@pytest.mark.parametrize("dim,group", SHAPES)
@pytest.mark.parametrize("shared,dtype", [(1, "bf16"), (7, "fp16"), (8, "bf16"), (16, "bf16"), (20, "fp16"), (33, "bf16")])
def test_attend(ops, dim, group, shared, dtype):
    r = np.random.default_rng(dim + shared)
    heads, page = 2, 16 if shared % 2 else 48
    row = -(-max(LENGTHS) // page)
    slots = page * (row + 9)
    cache, k, v = filled(ops, r, slots, page, heads, dim, group, dtype)
    table = np.stack([r.permutation(row + 9)[:row] for _ in LENGTHS]).astype(np.int32)
    q = cuda(r.standard_normal((len(LENGTHS), heads * shared, dim)), TYPES[dtype])
    check_attend(ops.AttendPlan(len(LENGTHS), heads * shared, heads, dim), q, cache, table, np.array(LENGTHS, dtype=np.int32), k, v)


@pytest.mark.parametrize("window,softcap,scale", [(1, 0.0, None), (7, 0.0, 0.3), (100, 0.0, None), (128, 5.0, None), (0, 30.0, 1.0), (0, 0.01, None)])
def test_windows_and_caps(ops, window, softcap, scale):
    r = np.random.default_rng(window)
    cache, k, v = filled(ops, r, 640, 32, 2, 128, 64, "bf16")
    table = np.stack([r.permutation(20)[:10] for _ in LENGTHS]).astype(np.int32)
    q = cuda(r.standard_normal((len(LENGTHS), 16, 128)), torch.bfloat16)
    plan = ops.AttendPlan(len(LENGTHS), 16, 2, 128, window=window, softcap=softcap, scale=scale)
    check_attend(plan, q, cache, table, np.array(LENGTHS, dtype=np.int32), k, v)


def test_holes_and_lengths_out_of_range(ops):
    r = np.random.default_rng(5)
    cache, k, v = filled(ops, r, 640, 16, 2, 64, 64, "fp16")
    table = np.stack([r.permutation(40)[:20] for _ in range(8)]).astype(np.int32)
    table[0, 3] = -1
    table[1, 0] = 40
    table[2] = -1
    table[3, :8] = 2**31 - 1
    table[4, 8:16] = -(2**31)
    lens = np.array([300, 300, 320, 129, 320, -4, 2**31 - 1, 321], dtype=np.int32)
    q = cuda(r.standard_normal((8, 6, 64)), torch.float16)
    out, lse = check_attend(ops.AttendPlan(8, 6, 2, 64), q, cache, table, lens, k, v)
    assert not out[2].any() and torch.isneginf(lse[2]).all() and not out[5].any()


@pytest.mark.parametrize("fill", [0, 255, 127])
def test_what_lies_behind_the_end_may_be_anything(ops, fill):
    """Only the tokens in use are written; the rest of their cells and pages is NaN, large or zero."""
    r = np.random.default_rng(fill)
    lens = np.array([1, 5, 16, 17, 40, 63], dtype=np.int32)
    page, heads, dim = 64, 2, 128
    cache = ops.PackedCache.zeros(6, page, heads, dim)
    cache.data.fill_(fill)
    x = cuda(r.standard_normal((2, 6 * page, heads, dim)), torch.bfloat16)
    used = np.concatenate([i * page + np.arange(n) for i, n in enumerate(lens)]).astype(np.int32)
    cache.write(x[0][used], x[1][used], cuda(used))
    q = cuda(r.standard_normal((6, 8, dim)), torch.bfloat16)
    check_attend(ops.AttendPlan(6, 8, heads, dim), q, cache, np.arange(6, dtype=np.int32)[:, None], lens, ref.quantise(f64(x[0]), 64), ref.quantise(f64(x[1]), 64))


@pytest.mark.parametrize("heads,shared,dim,group", [(1, 8, 128, 32), (8, 4, 128, 64), (2, 16, 64, 64), (1, 8, 256, 64), (3, 1, 96, 32)])
def test_long_requests_are_joined(ops, heads, shared, dim, group):
    """One request that every block has a part of, short ones before and behind it; the answer does not depend on who joins."""
    r = np.random.default_rng(heads)
    page = 64
    tokens = 70_000 // heads
    row = -(-tokens // page)
    cache, k, v = filled(ops, r, 2048, page, heads, dim, group, "bf16")
    lens = np.array([3, tokens, 900, 0, 1], dtype=np.int32)
    table = r.integers(0, 32, (5, row)).astype(np.int32)  # the same pages over and over
    q = cuda(r.standard_normal((5, heads * shared, dim)), torch.bfloat16)
    plan = ops.AttendPlan(5, heads * shared, heads, dim)
    out, lse = check_attend(plan, q, cache, table, lens, k, v)
    for _ in range(20):
        again, lse_again = plan.attend(q, cache, cuda(table), cuda(lens), return_lse=True)
        assert torch.equal(again, out) and torch.equal(lse_again, lse)


def test_many_short_requests(ops):
    r = np.random.default_rng(8)
    n, heads = 700, 4
    cache, k, v = filled(ops, r, 2048, 16, heads, 128, 64, "bf16")
    lens = r.integers(0, 200, n).astype(np.int32)
    table = r.integers(0, 128, (n, 13)).astype(np.int32)
    q = cuda(r.standard_normal((n, heads * 4, 128)), torch.bfloat16)
    check_attend(ops.AttendPlan(n, heads * 4, heads, 128), q, cache, table, lens, k, v, some=range(0, n, 13))


def test_weights_far_apart(ops):
    """A token that has nearly all the weight and nothing to say: the others, down to 2^-25 of it, still make the answer; and values
    whose sizes differ by many powers of 2 from token to token."""
    r = np.random.default_rng(9)
    tokens, dim = 256, 128
    k, v = np.zeros((tokens, 1, dim)), r.standard_normal((tokens, 1, dim))
    k[:, 0, 0] = -17.0 + r.integers(0, 2, tokens)
    k[37, 0, 0] = 0.0  # e^17 times the weight of the others
    v[37] = 0.0
    q = torch.zeros(1, 8, dim, device="cuda", dtype=torch.float16)
    q[:, :, 0] = 1.0
    table, lens = np.arange(4, dtype=np.int32)[None], np.array([tokens], dtype=np.int32)
    plan = ops.AttendPlan(1, 8, 1, dim, scale=1.0)
    cache, *held = filled(ops, r, tokens, 64, 1, dim, 64, "fp16", k=k, v=v)
    out, _ = check_attend(plan, q, cache, table, lens, *held)
    want = ref.attend(f64(q)[0], *held, np.arange(tokens), 1.0)[0]
    assert (np.abs(want) < 1e-4).all() and np.abs(f64(out)[0] - want).max() <= 2.0**-10 * np.abs(want).max() + 2.0**-25
    v = r.standard_normal((tokens, 1, dim)) * 2.0 ** r.integers(-60, 60, (tokens, 1, 1))
    cache, *held = filled(ops, r, tokens, 64, 1, dim, 32, "bf16", k=k, v=v)
    check_attend(plan, q.to(torch.bfloat16), cache, table, lens, *held)


@pytest.mark.parametrize("spread", [1.0, 6.0, 20.0])
def test_scores_of_every_spread(ops, spread):
    r = np.random.default_rng(int(spread))
    cache, k, v = filled(ops, r, 1024, 16, 2, 128, 64, "bf16")
    table = np.stack([r.permutation(64) for _ in range(4)]).astype(np.int32)
    q = cuda(r.standard_normal((4, 16, 128)) * spread, torch.bfloat16)
    q[1, 3] = 0.0
    q[2, 5, 1:] *= 2.0**-20
    q[3, 0] *= 2.0**100
    q[3, 1] *= 2.0**-100
    q[3, 0, :] = q[3, 0, :] * 0 + 2.0**-30
    check_attend(ops.AttendPlan(4, 16, 2, 128), q, cache, table, np.array([1024, 1000, 512, 77], dtype=np.int32), k, v)


def test_nan_goes_where_it_belongs(ops):
    r = np.random.default_rng(11)
    x = cuda(r.standard_normal((2, 64, 1, 128)), torch.bfloat16)
    x[1, 5, 0, 40] = float("nan")  # a group of V
    cache = ops.PackedCache.zeros(4, 16, 1, 128, group=32)
    cache.write(x[0], x[1], torch.arange(64, device="cuda", dtype=torch.int32))
    q = cuda(r.standard_normal((3, 8, 128)), torch.bfloat16)
    table = torch.arange(4, device="cuda", dtype=torch.int32)[None].expand(3, 4).contiguous()
    plan = ops.AttendPlan(3, 8, 1, 128)
    out = plan.attend(q, cache, table, torch.tensor([64, 5, 6], device="cuda", dtype=torch.int32))
    assert out[[0, 2]][..., 32:64].isnan().all() and not out[[0, 2]][..., :32].isnan().any() and not out[[0, 2]][..., 64:].isnan().any()
    assert not out[1].isnan().any()


def test_strided_q_and_out(ops):
    r = np.random.default_rng(12)
    cache, k, v = filled(ops, r, 320, 32, 2, 64, 32, "bf16")
    table, lens = np.stack([r.permutation(10) for _ in range(3)]).astype(np.int32), np.array([320, 200, 7], dtype=np.int32)
    plan = ops.AttendPlan(5, 8, 2, 64)
    fused = cuda(r.standard_normal((3, 8, 131)), torch.bfloat16)
    q = fused[..., 1:65]  # rows at odd elements
    out, _ = check_attend(plan, q, cache, table, lens, k, v)
    held = torch.full((3, 8, 67), 9.0, device="cuda", dtype=torch.bfloat16)
    plan.attend(q, cache, cuda(table), cuda(lens), out=held[..., 2:66])
    assert torch.equal(held[..., 2:66], out) and (held[..., :2] == 9).all() and (held[..., 66:] == 9).all()


def test_one_plan_for_both_kinds_of_cache(ops):
    r = np.random.default_rng(13)
    n, heads, dim = 6, 2, 128
    packed, k, v = filled(ops, r, 4096, 16, heads, dim, 64, "bf16")
    pages = torch.randn(2, 256, 16, heads, dim, device="cuda", dtype=torch.bfloat16)
    plain = ops.PagedCache(pages[0], pages[1])
    table, lens = np.stack([r.permutation(256) for _ in range(n)]).astype(np.int32), np.array([4096, 1, 0, 2000, 129, 3000], dtype=np.int32)
    q = cuda(r.standard_normal((n, 16, dim)), torch.bfloat16)
    plan = ops.AttendPlan(n, 16, heads, dim)
    first = plan.attend(q, plain, cuda(table), cuda(lens))
    check_attend(plan, q, packed, table, lens, k, v)
    assert torch.equal(plan.attend(q, plain, cuda(table), cuda(lens)), first)


def test_refused_calls_on_the_device(ops):
    cache = ops.PackedCache.zeros(4, 16, 2, 64)
    with pytest.raises(ValueError, match="float32"):
        cache.read(torch.zeros(1, device="cuda", dtype=torch.int32), dtype=torch.int8)
    with pytest.raises(ValueError, match="heads"):
        cache.write(torch.zeros(1, 3, 64, device="cuda", dtype=torch.bfloat16), torch.zeros(1, 3, 64, device="cuda", dtype=torch.bfloat16),
                    torch.zeros(1, device="cuda", dtype=torch.int32))
    with pytest.raises(ValueError, match="16 bytes"):
        ops.PackedCache(torch.zeros(ops.PackedCache.page_bytes(16, 64) + 8, device="cuda", dtype=torch.uint8)[8:].view(1, 1, -1), 16, 64)
    with pytest.raises(ValueError, match="slots"):
        cache.read(torch.zeros(2, 2, device="cuda", dtype=torch.int32))
    with pytest.raises(ValueError, match="other heads"):
        ops.AttendPlan(1, 4, 2, 128).attend(torch.zeros(1, 4, 128, device="cuda", dtype=torch.bfloat16), cache, torch.zeros(1, 1, device="cuda", dtype=torch.int32),
                                            torch.zeros(1, device="cuda", dtype=torch.int32))
    q = torch.zeros(1, 4, 64, device="cuda", dtype=torch.bfloat16, requires_grad=True)
    kv = torch.zeros(1, 2, 64, device="cuda", dtype=torch.bfloat16)
    zero = torch.zeros(1, device="cuda", dtype=torch.int32)
    out = ops.RopePlan(64).append(q, kv, kv, zero, zero, cache)
    with pytest.raises(RuntimeError, match="not differentiable"):
        out.sum().backward()
    out = ops.AttendPlan(1, 4, 2, 64).attend(q, cache, zero[None], zero + 1)
    with pytest.raises(RuntimeError, match="not differentiable"):
        out.sum().backward()


def test_a_decoding_step_in_a_graph_and_on_another_stream(ops):
    """Pages, append and attention over a cache of 4 bits, captured once and replayed with new tokens, against the definition."""
    r = np.random.default_rng(14)
    torch.manual_seed(14)
    n, q_heads, heads, dim, page, group, row = 5, 8, 2, 128, 16, 64, 8
    one = dict(dtype=torch.int32, device="cuda")
    table, free = torch.full((n, row), -1, **one), torch.randperm(n * row, device="cuda").to(torch.int32)
    seq, count, new = torch.zeros(n, **one), torch.tensor([n * row], **one), torch.tensor([1, 1, 0, 1, 1], **one)
    rope, plan, cache = ops.RopePlan(dim), ops.AttendPlan(n, q_heads, heads, dim), ops.PackedCache.zeros(n * row, page, heads, dim, group=group)
    fused = torch.zeros(n, q_heads + 2 * heads, dim, device="cuda", dtype=torch.bfloat16)

    def step():
        s = ops.pages_extend(new, seq, table, free, count, page, n)
        q = rope.append(fused[:, :q_heads], fused[:, q_heads : q_heads + heads], fused[:, q_heads + heads :], s.positions, s.slots, cache)
        rows = torch.zeros(n + 1, q_heads, dim, device="cuda", dtype=q.dtype)
        rows[torch.where(s.requests < 0, n, s.requests).long()] = q
        out = plan.attend(rows[:n], cache, table, s.seq_lens)
        seq.copy_(s.seq_lens)
        count.copy_(s.free_count)
        return rows, out, s

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    kept = seq.clone(), count.clone(), table.clone()
    with torch.cuda.stream(side):
        step()
        for a, b in zip((seq, count, table), kept):
            a.copy_(b)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rows, out, s = step()
    ks, vs = {i: [] for i in range(n)}, {i: [] for i in range(n)}
    freq = [10000.0 ** (-2.0 * i / dim) for i in range(dim // 2)]
    for t in range(40):
        fused.copy_(torch.randn_like(fused))
        graph.replay()
        x = f64(fused)
        for j, i in enumerate([0, 1, 3, 4]):
            turned = serve_ref.rotate(x[j : j + 1, q_heads : q_heads + heads], np.array([[t]]), freq, [0] * 64, "half")
            ks[i].append(turned[0])
            vs[i].append(x[j, q_heads + heads :])
    torch.cuda.synchronize()
    for i in range(n):
        if not ks[i]:
            assert not out[i].any()
            continue
        k, v = ref.quantise(np.stack(ks[i]), group), ref.quantise(np.stack(vs[i]), group)
        want, _, bound, _ = ref.attend(f64(rows)[i], k, v, np.arange(40), plan.scale)
        assert (np.abs(f64(out)[i] - want) <= bound + 2.0**-8 * (np.abs(want) + bound)).all()
    assert not plan.failed()


@pytest.mark.parametrize("scale", [0.0, -0.2, 1e-30])
def test_scales_of_either_sign(ops, scale):
    r = np.random.default_rng(15)
    cache, k, v = filled(ops, r, 320, 32, 2, 128, 64, "bf16")
    table, lens = np.stack([r.permutation(10) for _ in range(3)]).astype(np.int32), np.array([320, 200, 7], dtype=np.int32)
    q = cuda(r.standard_normal((3, 16, 128)), torch.bfloat16)
    q[1, 2] = 0.0
    check_attend(ops.AttendPlan(3, 16, 2, 128, scale=scale), q, cache, table, lens, k, v)
    check_attend(ops.AttendPlan(3, 16, 2, 128, scale=scale, softcap=3.0), q, cache, table, lens, k, v)


def test_two_plans_on_two_streams(ops):
    r = np.random.default_rng(16)
    cache, k, v = filled(ops, r, 4096, 16, 4, 128, 32, "bf16")
    table, lens = cuda(np.stack([r.permutation(256) for _ in range(20)]).astype(np.int32)), cuda(r.integers(0, 4097, 20).astype(np.int32))
    q = cuda(r.standard_normal((20, 32, 128)), torch.bfloat16)
    plans, streams = [ops.AttendPlan(20, 32, 4, 128) for _ in range(2)], [torch.cuda.Stream() for _ in range(2)]
    want = plans[0].attend(q, cache, table, lens)
    torch.cuda.synchronize()
    got = []
    for i in range(40):
        got.append(plans[i % 2].attend(q, cache, table, lens, stream=streams[i % 2]))
        got.append(plans[i % 2].attend(q, cache, table, lens, stream=streams[1 - i % 2]))  # ordered by the plan
    torch.cuda.synchronize()
    assert all(torch.equal(x, want) for x in got) and not plans[0].failed() and not plans[1].failed()


def test_append_without_q(ops):
    x = torch.randn(20, 2, 128, device="cuda", dtype=torch.float16)
    slots, positions = torch.randperm(32, device="cuda")[:20].to(torch.int32), torch.arange(20, device="cuda")
    cache, other = ops.PackedCache.zeros(2, 16, 2, 128), ops.PackedCache.zeros(2, 16, 2, 128)
    out = ops.RopePlan(128).append(x[:, :0], x, x, positions, slots, cache)
    ops.RopePlan(128).append(x, x, x, positions, slots, other)
    assert out.shape == (20, 0, 128) and torch.equal(cache.data, other.data)


@pytest.mark.parametrize("dim,group,dtype,heavy", [(128, 64, "bf16", False), (128, 64, "bf16", True), (128, 32, "fp16", True), (64, 64, "bf16", False),
                                                  (96, 32, "fp16", False), (256, 64, "bf16", True), (256, 32, "fp16", False)])
def test_scores_are_as_good_as_in_32_bits(ops, dim, group, dtype, heavy):
    """lse is off by 4 units of 2^-24 of the terms' size (their root sum of squares, of the largest score), root mean square.  A group's
    sum of products is cut off after each 16 elements, by half a unit in 2^-23 on average, where the sum so far is two thirds of
    its size on average: 0.4 units of 2^-24 each time, 1.5 for the four of a group of 64.  The groups' additions, the scale, the
    exponentials and the logarithm are as many roundings again as a sum in 32 bits has: 2.5."""
    r = np.random.default_rng(dim + group)
    heads, page, tokens = 2, 16, 640
    k = r.standard_normal((tokens, heads, dim))
    k[..., 5] *= 16 if heavy else 4
    if heavy:
        k += r.standard_normal((heads, dim)) ** 3
    cache, held_k, held_v = filled(ops, r, tokens, page, heads, dim, group, dtype, k=k)
    lens = np.array([640, 500, 33, 1, 17, 300, 128, 64], dtype=np.int32)
    table = np.stack([r.permutation(tokens // page) for _ in lens]).astype(np.int32)
    q = cuda(r.standard_normal((len(lens), 16, dim)), TYPES[dtype])
    plan = ops.AttendPlan(len(lens), 16, heads, dim)
    _, lse = check_attend(plan, q, cache, table, lens, held_k, held_v)
    codes, low, step = held_k
    values = (low[..., None] + step[..., None] * codes.reshape(*low.shape, group)).reshape(codes.shape)
    off = []
    for i, n in enumerate(lens):
        t = np.arange(n)
        at, x = table[i, t // page] * page + t % page, f64(q)[i]
        want = ref.attend(x, held_k, held_v, at, plan.scale)[1]
        terms = np.repeat(values[at], 8, axis=1) * x[None]  # [tokens, q heads, dim]
        size = np.sqrt((terms**2).sum(-1)).max(0) * plan.scale
        off.append((lse[i].cpu().double().numpy() - want) / np.maximum(size, 1.0))
    assert np.sqrt(np.mean(np.square(off))) <= 4 * 2.0**-24


@pytest.mark.parametrize("group", [32, 64])
@pytest.mark.parametrize("size", [2.0**40, 2.0**58, -(2.0**70), 2.0**100, -(2.0**120)])
@pytest.mark.parametrize("rise", [0.0, 0.05, 2.0])
def test_constant_values_behind_zeros(ops, group, size, rise):
    """Groups of one value have no step: the weight that they have is their value's.  Zeros, then large values, with scores that
    stay as they are or rise."""
    r = np.random.default_rng(17)
    tokens, dim = 512, 128
    k, v = np.zeros((tokens, 1, dim)), np.zeros((tokens, 1, dim))
    k[:, 0, 0] = np.maximum(0, np.arange(tokens) - 64) * rise / 4
    v[128:] = size
    v[300:, :, dim // 2 :] = size / 2.0**20  # the second half's values grow smaller on the way
    v[400:420] = 0.0
    cache, *held = filled(ops, r, tokens, 64, 1, dim, group, "bf16", k=k, v=v)
    q = torch.zeros(3, 8, dim, device="cuda", dtype=torch.bfloat16)
    q[:, :, 0] = torch.tensor([1.0, 0.5, 0.0, 2.0, -1.0, 0.25, 4.0, 1.0], device="cuda")
    table = np.stack([np.arange(8), np.arange(8), np.arange(8)[::-1]]).astype(np.int32)
    check_attend(ops.AttendPlan(3, 8, 1, dim, scale=1.0), q, cache, table, np.array([512, 140, 500], dtype=np.int32), *held)


@pytest.mark.parametrize("group", [32, 64])
@pytest.mark.parametrize("apart", [10, 18, 26])
def test_groups_of_values_far_apart(ops, group, apart):
    """The second half of a head has values 2^-apart of the first's: they are right to 15 / 2 x 2^-25 / 2^9 of the first's for each token
    (codes of at most 15, half of fp16's smallest step, the largest weight at 2^9 or more), and to 16 bits where that is far below."""
    r = np.random.default_rng(apart)
    tokens, dim = 256, 128
    v = r.standard_normal((tokens, 1, dim))
    v[..., dim // 2 :] *= 2.0**-apart
    for dtype, spread in (("bf16", 0.0), ("bf16", 1.0), ("fp16", 0.0)):
        if dtype == "fp16" and apart > 10:
            continue  # fp16 has no such numbers
        k = r.standard_normal((tokens, 1, dim)) * spread
        cache, held_k, held_v = filled(ops, r, tokens, 32, 1, dim, group, dtype, k=k, v=v)
        q = cuda(r.standard_normal((2, 8, dim)), TYPES[dtype])
        table, lens = np.stack([r.permutation(8) for _ in range(2)]).astype(np.int32), np.array([256, 199], dtype=np.int32)
        plan = ops.AttendPlan(2, 8, 1, dim)
        out, _ = check_attend(plan, q, cache, table, lens, held_k, held_v)
        for i, n in enumerate(lens):
            t = np.arange(n)
            want, _, bound, _ = ref.attend(f64(q)[i], held_k, held_v, table[i, t // 32] * 32 + t % 32, plan.scale)
            off, size = np.abs(f64(out)[i] - want)[:, dim // 2 :], np.abs(want)[:, dim // 2 :]
            # a score's error moves a weight, of values of up to 6 (and the softmax's, beside 2^-apart, is the same for both halves)
            own = (4 * 2.0**-20 + 2.0**-8 * (dtype == "bf16") + 2.0**-11 * (dtype == "fp16")) * size + 2.0**-apart * 6 * 2.0**-15
            assert (off <= own + 7.5 * 2.0**-34 * 6).all(), (dtype, i, (off / own).max())


def test_values_of_every_size(ops):
    """From 2^-105 to 2^120, all of one size, and from token to token."""
    r = np.random.default_rng(18)
    tokens, dim = 512, 128
    k = r.standard_normal((tokens, 1, dim))
    q = cuda(r.standard_normal((1, 8, dim)), torch.bfloat16)
    table, lens = np.arange(8, dtype=np.int32)[None], np.array([tokens], dtype=np.int32)
    plan = ops.AttendPlan(1, 8, 1, dim)
    for low, high in ((-105, -105), (-80, -80), (-40, -40), (23, 25), (60, 60), (118, 118), (-105, 60), (-60, 118), (-20, 30)):
        v = r.standard_normal((tokens, 1, dim)) * 2.0 ** r.integers(low, high + 1, (tokens, 1, 1))
        cache, *held = filled(ops, r, tokens, 64, 1, dim, 64, "bf16", k=k, v=v)
        check_attend(plan, q, cache, table, lens, *held)
        v = np.sort(np.abs(v), axis=0)  # growing, so that the scale is renewed on the way
        cache, *held = filled(ops, r, tokens, 64, 1, dim, 32, "bf16", k=k, v=v)
        check_attend(plan, q, cache, table, lens, *held)
