"""What the serving operators' arithmetic keeps where a sum or a difference shows it, against definitions in 64 bits."""
import math

import numpy as np
import pytest

import serve_ref as ref

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "e4m3": torch.float8_e4m3fn}


@pytest.fixture(scope="module")
def ops():
    from paper_2002_12798_b200 import ops

    return ops


def f64(t):
    return t.to(torch.float32).cpu().double().numpy()


@pytest.mark.parametrize("dtype,cache_dtype", [("bf16", "bf16"), ("fp16", "fp16"), ("bf16", "e4m3")])
@pytest.mark.parametrize("dim,group", [(64, 8), (128, 8), (256, 4), (128, 16)])
def test_attend_keeps_what_two_opposite_values_leave_over(ops, dim, group, dtype, cache_dtype):
    """Two tokens with V of opposite signs and weights that differ little: the output shows the weights' own error.  q has one
    element, so that scores are exact but for their scale, its product with log2 e and the subtraction of the maximum, 2^-24
    each of less than 1: p is within 2^-21 for that and 2^-22 for the power of two, either of the two tokens'."""
    n = 64
    r = np.random.default_rng(dim + group)
    k = np.zeros((n, 16, 1, dim))
    v = r.choice([0.5, 1.0, 1.5, 2.0], (n, 16, 1, dim))
    v[:, 1] = -v[:, 0]
    q = np.zeros((n, group, dim))
    q[:, :, 1] = r.integers(1, 9, (n, group)) / 8192.0
    k[:, 0, 0, 1], k[:, 1, 0, 1] = 0.5, -r.integers(1, 16, n) / 128.0  # scores apart by 2^-14 .. 2^-10
    table, lens = np.arange(n, dtype=np.int32)[:, None], np.full(n, 2, dtype=np.int32)
    held = [torch.from_numpy(x).float().cuda().to(TYPES[cache_dtype]) for x in (k, v)]
    qq = torch.from_numpy(q).float().cuda().to(TYPES[dtype])
    out = ops.AttendPlan(n, group, 1, dim, scale=1.0).attend(qq, ops.PagedCache(*held), torch.from_numpy(table).cuda(), torch.from_numpy(lens).cuda())
    want, _, _, mass = ref.attend(f64(qq), f64(held[0]), f64(held[1]), table, lens, 1.0)
    off = np.abs(f64(out) - want)
    assert (off <= ref.UNIT[dtype] * np.abs(want) + 2.0**-20 * mass).all(), (off / mass).max()


@pytest.mark.parametrize("dtype,cache_dtype", [("fp16", "fp16"), ("bf16", "e4m3"), ("bf16", "bf16")])
@pytest.mark.parametrize("dim,group", [(64, 8), (128, 1), (128, 16), (256, 8)])
@pytest.mark.parametrize("where", ["first", "middle", "every 61st", "some heads"])
def test_attend_beside_a_token_with_nearly_all_the_weight(ops, dim, group, where, dtype, cache_dtype):
    """One token's score stands 4 to 40 above all others' and its V is zero: the output is what the others have, and every
    one of them counts.  A score is the product of single elements, exact but for its scale and the subtraction of the
    maximum: 3 roundings of 2^-24 of at most 40 log2 e, so p is within 2^-17 of itself; requests are many, so that a warp
    meets most of a request's tokens behind its one."""
    gaps = [4, 8, 11, 12, 14, 16, 18, 20, 22, 24, 28, 32, 40]
    n, tokens, page = 13 * 25, 1500, 16
    row = -(-tokens // page)
    shape = (2 * row, page, 1, dim)
    k, v = torch.zeros(shape), torch.full(shape, 448.0 if cache_dtype == "e4m3" else 1024.0)
    r = np.random.default_rng(dim)
    at = {"first": [0], "middle": [777], "every 61st": range(0, tokens, 61), "some heads": [3]}[where]
    flat_k, flat_v = k.view(-1, dim), v.view(-1, dim)
    for t in at:
        flat_k[t, 0], flat_v[t] = 1.0, 0.0
    k.view(2, -1, dim)[1].copy_(k.view(2, -1, dim)[0])  # the second half: the others differ in scores, up to 2 either way
    k.view(2, -1, dim)[1][:, 1] = torch.from_numpy(r.integers(-8, 9, row * page) / 8.0)
    v.view(2, -1, dim)[1].copy_(v.view(2, -1, dim)[0])
    q = torch.zeros(n, group, dim)
    q[:, :, 0] = torch.tensor(gaps * 25)[:, None]
    if where == "some heads":
        q[:, ::3, 0] = 0.0
    q[:, :, 1] = 1.0
    table = np.arange(2 * row, dtype=np.int32).reshape(2, row)[np.arange(n) % 2]
    lens = np.full(n, tokens, dtype=np.int32) - np.arange(n, dtype=np.int32) % 7
    held = [x.cuda().to(TYPES[cache_dtype]) for x in (k, v)]
    qq = q.cuda().to(TYPES[dtype])
    args = qq, ops.PagedCache(*held), torch.from_numpy(table).cuda(), torch.from_numpy(lens).cuda()
    out, lse = ops.AttendPlan(n, group, 1, dim, scale=1.0).attend(*args, return_lse=True)
    some = np.arange(0, n, 4)
    want, want_lse, _, mass = ref.attend(f64(qq)[some], f64(held[0]), f64(held[1]), table[some], lens[some], 1.0)
    off = np.abs(f64(out)[some] - want)
    # half of fp16's smallest step, where the output is that small
    assert (off <= ref.UNIT[dtype] * np.abs(want) + 2.0**-15 * mass + 2.0**-25).all(), (off / mass).max()
    assert (np.abs(f64(lse)[some] - want_lse) <= 2.0**-16 + 2.0**-22 * np.abs(want_lse)).all()


@pytest.mark.parametrize("dim,group", [(64, 8), (128, 16), (256, 3)])
def test_attend_infinity_beside_a_token_with_nearly_all_the_weight(ops, dim, group):
    """An infinity in V is one in the output however small its token's weight is (as far as 32 bits hold that), and nothing
    else; what lies behind a request's end is not."""
    n, tokens, page = 40, 200, 16
    k, v = torch.zeros(13, page, 1, dim), torch.ones(13, page, 1, dim)
    k.view(-1, dim)[5, 0] = 1.0
    v.view(-1, dim)[[4, 100], [3, 7]] = math.inf
    v.view(-1, dim)[150, 9] = -math.inf
    v.view(-1, dim)[tokens:] = math.nan
    q = torch.zeros(n, group, dim)
    q[:, :, 0] = torch.arange(n)[:, None]
    table = torch.arange(13, dtype=torch.int32).repeat(n, 1).cuda()
    held = [x.cuda().half() for x in (k, v)]
    out = f64(ops.AttendPlan(n, group, 1, dim, scale=1.0).attend(q.cuda().half(), ops.PagedCache(*held), table, torch.full((n,), tokens, dtype=torch.int32).cuda()))
    for at, value in ((3, math.inf), (7, math.inf), (9, -math.inf)):
        assert (out[..., at] == value).all()
    rest = np.delete(out, [3, 7, 9], 2)
    assert (np.abs(rest - 1) <= 2.0**-11).all()


@pytest.mark.parametrize("dtype,cache_dtype", [("fp16", "fp16"), ("bf16", "e4m3")])
@pytest.mark.parametrize("spread", [1.0, 8.0, 40.0])
def test_attend_scores_far_apart_everywhere(ops, spread, dtype, cache_dtype):
    """Random scores of up to some hundreds of powers of two apart: within the bound of a 32-bit computation."""
    torch.manual_seed(int(spread))
    r = np.random.default_rng(int(spread))
    n, heads, dim, page = 24, 2, 128, 16
    lens = r.integers(1, 700, n).astype(np.int32)
    table = r.permutation(n * 44).astype(np.int32).reshape(n, 44)
    k, v = (torch.randn(n * 44, page, heads, dim, device="cuda").to(TYPES[cache_dtype]) for _ in range(2))
    q = (torch.randn(n, 16, dim, device="cuda") * spread).to(TYPES[dtype])
    plan = ops.AttendPlan(n, 16, heads, dim)
    out, lse = plan.attend(q, ops.PagedCache(k, v), torch.from_numpy(table).cuda(), torch.from_numpy(lens).cuda(), return_lse=True)
    want, want_lse, size, mass = ref.attend(f64(q), f64(k), f64(v), table, lens, plan.scale)
    bound, lse_bound = ref.attend_bound(want, size, mass, dim, dtype)
    assert (np.abs(f64(out) - want) <= bound).all()
    assert (np.abs(f64(lse) - want_lse) <= lse_bound + 2.0**-22 * np.abs(want_lse)).all()


@pytest.mark.parametrize("dtype,cache_dtype", [("fp16", "fp16"), ("bf16", "bf16"), ("bf16", "e4m3")])
@pytest.mark.parametrize("softcap", [1e-40, 1e-6, 0.5, 5.0, 30.0, 50.0, 1e3, 1e5, 1e8, 1e30])
def test_attend_softcap_of_any_size(ops, softcap, dtype, cache_dtype):
    """A score that the cap hardly touches is what it is without one: the bound is that of a score in 32 bits, of which the
    hyperbolic tangent adds 2^-20 of itself (the bound has 16 times 2^-23 to spare for such)."""
    torch.manual_seed(3)
    r = np.random.default_rng(3)
    n, heads, dim, page = 12, 2, 64, 16
    lens = r.integers(1, 300, n).astype(np.int32)
    table = r.permutation(n * 19).astype(np.int32).reshape(n, 19)
    k, v = (torch.randn(n * 19, page, heads, dim, device="cuda").to(TYPES[cache_dtype]) for _ in range(2))
    q = torch.randn(n, 8, dim, device="cuda").to(TYPES[dtype])
    q[0], q[1] = 0.0, q[1] * 1e-3
    plan = ops.AttendPlan(n, 8, heads, dim, softcap=softcap)
    out, lse = plan.attend(q, ops.PagedCache(k, v), torch.from_numpy(table).cuda(), torch.from_numpy(lens).cuda(), return_lse=True)
    cap = float(np.float32(softcap))
    want, want_lse, size, mass = ref.attend(f64(q), f64(k), f64(v), table, lens, plan.scale, softcap=cap)
    bound, lse_bound = ref.attend_bound(want, size, mass, dim, dtype)
    off = np.abs(f64(out) - want) / bound
    assert (off <= 1).all(), off.max()
    assert (np.abs(f64(lse) - want_lse) <= lse_bound + 2.0**-22 * np.abs(want_lse)).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("power", [10, 16, 20, 26])
def test_attend_query_elements_far_apart_over_8_bits(ops, power, dtype):
    """One element of q is 2^power of the others and meets zeros in K: the others count in full."""
    torch.manual_seed(power)
    r = np.random.default_rng(power)
    n, heads, dim, page = 6, 2, 128, 16
    lens = r.integers(1, 300, n).astype(np.int32)
    table = r.permutation(n * 19).astype(np.int32).reshape(n, 19)
    k, v = (torch.randn(n * 19, page, heads, dim, device="cuda") for _ in range(2))
    k[..., 5] = 0.0
    held = [x.to(TYPES["e4m3"]) for x in (k, v)]
    small = 2.0 ** (15 - power) if dtype == "fp16" else 1.0
    q = (torch.rand(n, 8, dim, device="cuda") + 1) * small * torch.where(torch.rand(n, 8, dim, device="cuda") < 0.5, -1.0, 1.0)
    q[..., 5] = small * 2.0**power * 1.5
    q = q.to(TYPES[dtype])
    assert torch.isfinite(q).all()
    plan = ops.AttendPlan(n, 8, heads, dim, scale=0.2 / small)
    out, lse = plan.attend(q, ops.PagedCache(*held), torch.from_numpy(table).cuda(), torch.from_numpy(lens).cuda(), return_lse=True)
    want, want_lse, size, mass = ref.attend(f64(q), f64(held[0]), f64(held[1]), table, lens, float(np.float32(plan.scale)))
    bound, lse_bound = ref.attend_bound(want, size, mass, dim, dtype)
    off = np.abs(f64(out) - want) / bound
    assert (off <= 1).all(), off.max()
    assert (np.abs(f64(lse) - want_lse) <= lse_bound + 2.0**-22 * np.abs(want_lse)).all()


@pytest.mark.parametrize("scale", [1.0 / 64, 3.0, 0.7, 1.3, 7.0 / 1024, 11.0, 13.0 / 8, 57.0, 113.0 / 64, 2.0**-126, 2.0**-130, 1e-39, 2.0**-149, 3e38])
def test_append_divides_by_the_scale(ops, scale):
    """Every bf16 value and some fp16 ones into an e4m3 cache: the quotient in 32 bits, rounded; exactly."""
    s = np.float32(scale)
    every = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    x = every.view(256, 1, 256).cuda()
    k, v = (torch.zeros(2, 128, 1, 256, device="cuda").to(TYPES["e4m3"]) for _ in range(2))
    slots, pos = torch.arange(256, dtype=torch.int32, device="cuda"), torch.zeros(256, dtype=torch.int32, device="cuda")
    ops.RopePlan(256, 0).append(x, x, x, pos, slots, ops.PagedCache(k, v, k_scale=float(s), v_scale=float(s)))
    with np.errstate(all="ignore"):
        quotient = every.float().numpy() / s
    want = torch.from_numpy(np.clip(quotient, -448, 448)).to(TYPES["e4m3"]).view(torch.uint8).numpy().reshape(-1)
    nan = np.isnan(quotient)
    for got in (k, v):
        got = got.view(torch.uint8).cpu().numpy().reshape(-1)
        assert ((got[nan] & 0x7F) == 0x7F).all()
        assert np.array_equal(got[~nan], want[~nan]), (got[~nan] != want[~nan]).sum()


@pytest.mark.parametrize("base,first", [(10000.0, 0), (1e6, 100000), (10.0, -70)])
@pytest.mark.parametrize("pairs", ["half", "adjacent"])
def test_rotate_in_fp32_is_as_exact_as_rounded_cos_and_sin(ops, base, first, pairs):
    """Over half a million elements, against the same turn with cos and sin of 64 bits rounded once (a tenth more is allowed)."""
    torch.manual_seed(0)
    dim, tokens = 128, 1024
    half = dim // 2
    plan = ops.RopePlan(dim, base=base, pairs=pairs)
    pos = torch.arange(first, first + tokens, dtype=torch.int32, device="cuda")
    x = torch.randn(tokens, 4, dim, device="cuda")
    (y,) = plan.rotate([x], pos)
    angle = pos.double()[:, None] * torch.tensor([base ** (-2.0 * i / dim) for i in range(half)], dtype=torch.float64, device="cuda")
    cos, sin = angle.cos()[:, None], angle.sin()[:, None]
    a, b = (x[..., :half], x[..., half:]) if pairs == "half" else (x[..., 0::2], x[..., 1::2])
    got = (y[..., :half], y[..., half:]) if pairs == "half" else (y[..., 0::2], y[..., 1::2])
    want = torch.stack([a.double() * cos - b.double() * sin, b.double() * cos + a.double() * sin])
    c, s = cos.float(), sin.float()
    plain = torch.stack([a * c - b * s, b * c + a * s])
    off = lambda z: float((z.double() - want).norm() / want.norm())  # noqa: E731
    assert off(torch.stack(got)) <= 1.1 * off(plain), (off(torch.stack(got)), off(plain))


@pytest.mark.parametrize("dtype,cache_dtype", [("fp16", "fp16"), ("bf16", "e4m3"), ("bf16", "bf16")])
@pytest.mark.parametrize("dim,group,window,softcap", [(64, 32, 0, 0.0), (128, 29, 0, 0.0), (128, 40, 150, 0.0), (256, 17, 0, 40.0), (80, 20, 0, 1e4)])
def test_attend_many_q_heads_with_scores_far_apart(ops, dim, group, window, softcap, dtype, cache_dtype):
    """Groups of more than 16 q heads, the kernels with the most of them, over scores near together and far apart, with tokens
    that take no part in the same steps and pages that end inside them."""
    torch.manual_seed(dim + group)
    r = np.random.default_rng(dim + group)
    page = 24
    lens = np.array([0, 1, 33, 700, 64, 1500], dtype=np.int32)
    n, row = len(lens), -(-1500 // page)
    table = r.permutation(n * row).astype(np.int32).reshape(n, row)
    table[3, [0, 5, 6]] = -1
    k, v = (torch.randn(n * row, page, 2, dim, device="cuda").to(TYPES[cache_dtype]) for _ in range(2))
    q = torch.randn(n, 2 * group, dim, device="cuda")
    q[:, ::3] *= 12
    q[:, 1::5] *= 40
    q = q.to(TYPES[dtype])
    plan = ops.AttendPlan(n, 2 * group, 2, dim, window=window, softcap=softcap)
    out, lse = plan.attend(q, ops.PagedCache(k, v), torch.from_numpy(table).cuda(), torch.from_numpy(lens).cuda(), return_lse=True)
    want, want_lse, size, mass = ref.attend(f64(q), f64(k), f64(v), table, lens, plan.scale, window, softcap)
    bound, lse_bound = ref.attend_bound(want, size, mass, dim, dtype)
    off = np.abs(f64(out) - want) / bound
    assert (off <= 1).all(), off.max()
    there = np.isfinite(want_lse)
    assert np.array_equal(there, np.isfinite(f64(lse)))
    assert (np.abs(f64(lse)[there] - want_lse[there]) <= lse_bound[there] + 2.0**-22 * np.abs(want_lse[there])).all()
