"""Sampling on the GPU against its definition in 64 bits, row by row and token by token."""
import numpy as np
import pytest

import packed_ref as ref

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
NEAR = 2.0**-30  # in probability: how near to a border the definition's answer is not looked at (sums of weights of 2^-36)


@pytest.fixture(scope="module")
def ops():
    from paper_2002_12798_b200 import ops

    return ops


def check(ops, logits, u, **settings):
    token, logprob = ops.sample(logits, u, return_logprob=True, **settings)
    assert token.dtype == torch.int32 and logprob.dtype == torch.float32
    x, uu = logits.float().cpu().numpy().astype(np.float64), u.cpu().numpy()
    each = {n: (v.cpu().numpy() if isinstance(v, torch.Tensor) else np.full(len(x), np.float32(v) if n != "top_k" else v))
            for n, v in {"temperature": 1.0, "top_k": 0, "top_p": 1.0, "min_p": 0.0, **settings}.items()}
    skipped = 0
    for r in range(len(x)):
        want, want_logprob, near = ref.sample(x[r], uu[r], *(float(each[n][r]) if n != "top_k" else int(each[n][r]) for n in ("temperature", "top_k", "top_p", "min_p")))
        if near < NEAR and uu[r] > 0:
            skipped += 1
            continue
        assert int(token[r]) == want, (r, int(token[r]), want, near)
        got = float(logprob[r])
        assert got == want_logprob or abs(got - want_logprob) <= 2.0**-23 * abs(want_logprob) + 2.0**-30, (r, got, want_logprob)
    assert skipped <= len(x) // 50
    return token


SETTINGS = [dict(), dict(temperature=0.7), dict(temperature=1.7, top_k=40), dict(top_p=0.9), dict(top_p=0.5, temperature=3.0), dict(min_p=0.1),
            dict(temperature=0.8, top_k=50, top_p=0.95), dict(top_k=7, top_p=0.3, min_p=0.02), dict(temperature=0.0), dict(top_k=1), dict(top_p=0.0),
            dict(min_p=1.0), dict(top_k=10**6, top_p=0.999, temperature=20.0), dict(top_k=500, min_p=0.001)]


@pytest.mark.parametrize("settings", SETTINGS)
@pytest.mark.parametrize("rows,vocab,dtype", [(1, 1, "fp32"), (3, 2, "bf16"), (5, 33, "fp16"), (2, 1000, "fp32"), (1, 32000, "fp32"), (9, 50001, "bf16"), (200, 3001, "fp16")])
def test_sample(ops, settings, rows, vocab, dtype):
    g = torch.Generator(device="cuda").manual_seed(rows + vocab)
    x = (torch.randn(rows, vocab, generator=g, device="cuda") * 3).to(TYPES[dtype])
    check(ops, x, torch.rand(rows, generator=g, device="cuda"), **settings)


def test_large_vocabularies_of_each_cluster(ops):
    """1 to 300 rows: from eight blocks to a row down to one."""
    g = torch.Generator(device="cuda").manual_seed(1)
    for rows, vocab, dtype in [(1, 262144, "bf16"), (4, 200003, "fp32"), (20, 131072, "fp16"), (40, 65537, "fp32"), (90, 40001, "bf16"), (300, 9001, "fp32")]:
        x = (torch.randn(rows, vocab, generator=g, device="cuda") * 2).to(TYPES[dtype])
        u = torch.rand(rows, generator=g, device="cuda")
        for settings in (dict(), dict(top_p=0.9, temperature=0.8), dict(top_k=100, top_p=0.9)):
            check(ops, x, u, **settings)


def test_settings_by_row(ops):
    g = torch.Generator(device="cuda").manual_seed(2)
    rows, vocab = 300, 5003
    x = (torch.randn(rows, vocab, generator=g, device="cuda") * 3).bfloat16()
    pick = lambda values, dtype: torch.tensor(values, device="cuda", dtype=dtype)[torch.randint(0, len(values), (rows,), generator=g, device="cuda")]  # noqa: E731
    check(ops, x, torch.rand(rows, generator=g, device="cuda"), temperature=pick([0.0, 0.3, 1.0, 2.5, -1.0], torch.float32),
          top_k=pick([0, -1, 1, 5, 80, 5002, 5003, 9999], torch.int32), top_p=pick([1.0, 0.9, 0.5, 0.01], torch.float32), min_p=pick([0.0, 0.05, 0.5], torch.float32))


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
def test_ties(ops, dtype):
    """Few distinct logits: a bound falls among equal ones, of which the first by index are kept."""
    g = torch.Generator(device="cuda").manual_seed(3)
    rows, vocab = 40, 20011
    x = torch.randint(0, 4, (rows, vocab), generator=g, device="cuda").to(TYPES[dtype])
    x[0] = 1.5
    x[1] = -3.0
    u = torch.rand(rows, generator=g, device="cuda")
    for settings in (dict(), dict(top_k=100), dict(top_k=5001), dict(top_p=0.3), dict(top_p=0.9), dict(top_k=6000, top_p=0.7), dict(min_p=0.3, top_k=9000)):
        check(ops, x, u, **settings)


def test_logits_next_to_one_another(ops):
    """fp32 logits that differ in their last bits, and ones from zero up through all its exponents."""
    g = torch.Generator(device="cuda").manual_seed(4)
    u = torch.rand(6, generator=g, device="cuda")
    x = 7.0 + torch.randint(0, 3000, (6, 30000), generator=g, device="cuda") * 2.0**-21
    y = torch.exp2(-torch.rand(6, 30000, generator=g, device="cuda") * 140) * torch.where(torch.rand(6, 30000, generator=g, device="cuda") < 0.5, 1, -1)
    for z in (x, y, -x, torch.cat([x[:, :100], y], 1)):
        for settings in (dict(top_k=1000), dict(top_p=0.4), dict(top_k=20000, top_p=0.9)):
            check(ops, z.contiguous(), u, **settings)


def test_infinities_and_nan(ops):
    inf, nan = float("inf"), float("nan")
    x = torch.randn(9, 777, device="cuda")
    x[0] = -inf
    x[1] = nan
    x[2, ::3] = nan
    x[3, ::2] = -inf
    x[4, [5, 70, 700]] = inf
    x[5] = inf
    x[6, 5:] = -inf
    x[7] = torch.finfo(torch.float32).min
    x[8, 0], x[8, 1] = 3e38, -3e38
    for dtype in ("fp32", "bf16"):
        for u in (0.0, 0.4, 0.999):
            for settings in (dict(), dict(top_k=2), dict(top_p=0.5), dict(temperature=0.0), dict(min_p=0.5)):
                token = check(ops, x.to(TYPES[dtype]), torch.full((9,), u, device="cuda"), **settings)
                assert token[0] == -1 and token[1] == -1
    # what is masked by the type's lowest value is not drawn beside anything else
    y = torch.full((4, 1000), torch.finfo(torch.bfloat16).min, device="cuda", dtype=torch.bfloat16)
    y[:, 77] = 0.0
    assert ops.sample(y, torch.tensor([0.0, 0.3, 0.9, 1.0 - 2.0**-24], device="cuda")).tolist() == [77] * 4


def test_uniforms_at_and_beyond_their_ends(ops):
    x = torch.tensor([[-float("inf"), 1.0, 1.0, -float("inf"), 1.0, -float("inf")]], device="cuda").expand(7, 6).contiguous()
    u = torch.tensor([0.0, -1.0, float("nan"), 0.5, 1 - 2.0**-24, 1.0, 5.0], device="cuda")
    assert ops.sample(x, u).tolist() == [1, 1, 1, 2, 4, 4, 4]


def test_temperatures_of_every_size(ops):
    g = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn(8, 3000, generator=g, device="cuda") * 5
    u = torch.rand(8, generator=g, device="cuda")
    for t in (1e-40, 1e-6, 0.01, 50.0, 1e6, 1e30):
        for settings in (dict(), dict(top_k=30), dict(top_p=0.5)):
            check(ops, x, u, temperature=t, **settings)
    check(ops, x * 1e30, u, temperature=1e30)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_rows_of_any_alignment(ops, dtype):
    """Rows that begin at every element of a 16-byte piece, and what lies around them is not looked at."""
    g = torch.Generator(device="cuda").manual_seed(6)
    for offset in range(9):
        for stride in (2048, 2051):
            flat = torch.full((offset + 5 * stride + 64,), 1e4, device="cuda", dtype=TYPES[dtype])
            x = flat.as_strided((5, 2011), (stride, 1), offset)
            x.copy_(torch.randn(5, 2011, generator=g, device="cuda") * 3)
            check(ops, x, torch.rand(5, generator=g, device="cuda"), top_p=0.8, temperature=0.9)


def test_a_broadcast_row(ops):
    x = torch.randn(1, 5000, device="cuda", dtype=torch.float16) * 3
    check(ops, x.expand(50, 5000), torch.rand(50, device="cuda"), top_k=100)


def test_outputs_and_refusals(ops):
    x, u = torch.randn(4, 100, device="cuda"), torch.rand(4, device="cuda")
    out = torch.empty(4, device="cuda", dtype=torch.int32)
    assert ops.sample(x, u, out=out) is not None and torch.equal(out, ops.sample(x, u))
    assert ops.sample(x[:0], u[:0]).shape == (0,)
    for bad, why in [((x, u[:3]), "uniforms"), ((x, u.double()), "uniforms"), ((x.t(), u), "contiguous rows"), ((x[0], u), "contiguous rows")]:
        with pytest.raises(ValueError, match=why):
            ops.sample(*bad)
    for bad, why in [(dict(top_k=torch.zeros(4, device="cuda")), "int32"), (dict(temperature=torch.ones(3, device="cuda")), "float32"), (dict(out=out[:3]), "out")]:
        with pytest.raises(ValueError, match=why):
            ops.sample(x, u, **bad)
    from paper_2002_12798_b200.binding import AmapError

    for bad in (dict(top_p=1.5), dict(min_p=-0.1), dict(temperature=float("nan"))):
        with pytest.raises(AmapError):
            ops.sample(x, u, **bad)
    with pytest.raises(AmapError):
        ops.sample(x.double(), u)
    y = x.clone().requires_grad_()
    token, logprob = ops.sample(y, u, return_logprob=True)
    assert torch.equal(token, ops.sample(x, u))
    with pytest.raises(RuntimeError, match="not differentiable"):
        logprob.sum().backward()


def test_a_captured_call_on_another_stream(ops):
    x, u = torch.randn(6, 40000, device="cuda") * 2, torch.rand(6, device="cuda")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    ops.sample(x, u, top_p=0.9, stream=stream)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        token = ops.sample(x, u, top_p=0.9, top_k=300)
    for _ in range(3):
        x.copy_(torch.randn_like(x) * 2)
        u.copy_(torch.rand_like(u))
        graph.replay()
        assert torch.equal(token, ops.sample(x, u, top_p=0.9, top_k=300))


def test_drawn_as_often_as_their_weight(ops):
    """Many uniforms, evenly spaced, over one row: every token as often as its probability says, to within one."""
    x = torch.randn(1, 50, device="cuda") * 2
    n = 20000
    token = ops.sample(x.expand(n, 50), (torch.arange(n, device="cuda") + 0.5) / n, temperature=1.3)
    p = torch.softmax(x[0].double() / float(np.float32(1.3)), 0).cpu().numpy()
    assert np.abs(np.bincount(token.cpu().numpy(), minlength=50) - n * p).max() <= 1.0 + n * 2.0**-23


def test_settings_that_are_no_numbers_or_outside(ops):
    x, u = torch.randn(4, 3000, device="cuda") * 3, torch.rand(4, device="cuda")
    of = lambda *v: torch.tensor(v, device="cuda")  # noqa: E731
    nan = float("nan")
    plain = ops.sample(x, u)
    assert torch.equal(ops.sample(x, u, top_p=of(nan, 1.0, 2.0, nan), min_p=of(nan, 0.0, -1.0, 0.0)), plain)
    first = x.argmax(1).to(torch.int32)
    assert torch.equal(ops.sample(x, u, temperature=of(nan, 0.0, -2.0, -0.0)), first)
    assert torch.equal(ops.sample(x, u, top_p=of(-1.0, 0.0, -0.5, 1e-9), min_p=0.0), first)
    assert torch.equal(ops.sample(x, u, min_p=of(1.0, 7.0, float("inf"), 1.5)), first)


@pytest.mark.parametrize("rows,vocab", [(1, 200000), (30, 50000), (200, 20000)])
def test_top_k_of_every_size(ops, rows, vocab):
    """Bounds from a block's threads, from the row's, and none."""
    g = torch.Generator(device="cuda").manual_seed(vocab)
    for dtype in ("bf16", "fp32"):
        x = (torch.randn(rows, vocab, generator=g, device="cuda") * 2).to(TYPES[dtype])
        u = torch.rand(rows, generator=g, device="cuda")
        for k in (2, 63, 64, 65, 129, 512, 513, 1023, 1025, 4097, vocab - 1):
            check(ops, x[:3], u[:3], top_k=k)
            check(ops, x[-2:], u[-2:], top_k=k, top_p=0.7)
        token = ops.sample(x, u, top_k=100)
        assert torch.equal(token[-2:], ops.sample(x[-2:], u[-2:], top_k=100))  # however many blocks a row has


def test_flat_rows_keep_most_of_their_tokens(ops):
    """Lists overflow, bounds fall deep into the row; bf16 logits around zero share a bin."""
    g = torch.Generator(device="cuda").manual_seed(8)
    for rows, vocab in ((3, 150001), (160, 30011)):
        for spread in (0.01, 0.5):
            for dtype in ("bf16", "fp16", "fp32"):
                x = (torch.randn(rows, vocab, generator=g, device="cuda") * spread).to(TYPES[dtype])
                u = torch.rand(rows, generator=g, device="cuda")
                for settings in (dict(top_p=0.95), dict(top_p=0.4, temperature=0.3), dict(top_k=vocab // 2, top_p=0.9), dict(min_p=0.2, top_p=0.5)):
                    check(ops, x[:3], u[:3], **settings)
                    assert torch.equal(ops.sample(x, u, **settings)[:3], ops.sample(x[:3], u[:3], **settings))


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("shift,temperature", [(-20.0, 0.001), (-100.0, 0.01), (-512.0, 0.05), (-200.0, 0.1), (-9984.0, 1.0), (-9984.0, 0.3), (0.0, 1e-4), (100.0, 0.01)])
def test_largest_logits_below_zero(ops, dtype, shift, temperature):
    """The lowest number with a weight lies between two 16-bit logits, next to a negative largest one: what is smaller, a NaN and what
    lies outside the row have none.  Nothing cut off, min_p over more tokens than the lists hold, top_k of all; every row is written."""
    g = torch.Generator(device="cuda").manual_seed(7)
    for rows, vocab, offset in ((5, 3001, 0), (3, 20011, 3), (2, 777, 5)):
        stride = vocab + 6
        flat = torch.zeros(offset + rows * stride + 16, device="cuda", dtype=TYPES[dtype])
        x = flat.as_strided((rows, vocab), (stride, 1), offset)
        x.copy_(torch.randn(rows, vocab, generator=g, device="cuda") * 3 + shift)
        x[0, ::3] = float("nan")
        x[1, 1:] = -float("inf")
        u = torch.rand(rows, generator=g, device="cuda")
        for settings in (dict(), dict(min_p=1e-6), dict(top_k=vocab), dict(top_p=0.9), dict(top_k=vocab // 2, top_p=0.95)):
            check(ops, x, u, temperature=temperature, **settings)
            out = torch.full((rows,), -7, device="cuda", dtype=torch.int32)
            ops.sample(x, u, temperature=temperature, out=out, **settings)
            assert ((out >= 0) & (out < vocab)).all()


def test_rows_of_the_lowest_numbers(ops):
    """All of a row masked by the type's lowest number, with and without a NaN in it: the masked tokens share the weight."""
    for dtype in ("bf16", "fp16", "fp32"):
        for vocab in (1000, 1003, 30011):
            x = torch.full((4, vocab), torch.finfo(TYPES[dtype]).min, device="cuda", dtype=TYPES[dtype])
            x[2, ::2] = float("nan")
            x[3, : vocab - 1] = -float("inf")
            u = torch.tensor([0.1, 0.7, 0.6, 0.5], device="cuda")
            for settings in (dict(), dict(temperature=0.01), dict(temperature=30.0), dict(min_p=0.5), dict(top_k=vocab), dict(top_p=0.9)):
                check(ops, x, u, **settings)


def test_top_p_next_to_one_over_a_tail_of_few_units(ops):
    """What top_p leaves out is less than the rounding of the weights of the tail: a tail token of 3.6 units of 2^-44 counts as 4."""
    vocab = 1 << 19
    x = torch.full((1, vocab), float(np.log(3.6 * 2.0**-44)), device="cuda")
    x[0, 100::340] = float(np.log(2.0**-24))  # more than one block sorts, spread over the row
    x[0, 5], x[0, 400_000] = 0.0, float(np.log(0.85))
    x = x.expand(6, vocab)
    u = torch.tensor([0.1, 0.5, 0.54, 0.6, 0.9, 0.99], device="cuda")
    p = 1.0 - 2.0**-24
    for settings in (dict(top_p=p), dict(top_p=torch.full((6,), p, device="cuda"))):
        assert ops.sample(x, u, **settings).tolist() == [5, 5, 5, 400_000, 400_000, 400_000]


def test_temperatures_without_bound(ops):
    """Above 1e30 they count as that, an infinite one of a row, too; NaN and -infinity are not drawn at any of them."""
    rows = 6
    x = torch.zeros(rows, 1003, device="cuda")
    x[:, ::2] = float("nan")
    x[:, 1::4] = -float("inf")
    x[:, 3] = -3.3e38
    x[1] -= 3.2e38
    x[2] += 3.4e38
    x[3, 3::4] = -torch.arange(1, 251, device="cuda") * 1e30  # the tokens 3, 7, 11, ..
    x[4] = torch.finfo(torch.float32).min
    x[4, ::5] = float("nan")
    x[5] = torch.nextafter(x[4, 1], torch.tensor(0.0, device="cuda"))
    x[5, ::3] = -float("inf")
    u = torch.tensor([0.0213, 0.5077, 0.9713, 0.6071, 0.3019, 0.9037], device="cuda")
    inf = torch.full((rows,), float("inf"), device="cuda")
    for t in (1e29, 1e30, 1e35, 1e36, 3e38):
        for settings in (dict(), dict(top_k=100), dict(top_p=0.5), dict(min_p=1e-3)):
            want = ops.sample(x, u, temperature=min(t, 1e30), **settings)
            check(ops, x, u, temperature=min(t, 1e30), **settings)
            assert torch.equal(ops.sample(x, u, temperature=t, **settings), want)
            if t == 1e36:
                assert torch.equal(ops.sample(x, u, temperature=inf, **settings), want)


def test_probabilities_of_unlikely_tokens(ops):
    """A token of 2^-30 to 2^-44 of the largest one's weight, drawn because it comes first: the log of its probability is that of
    its logit, not of its weight in whole units."""
    for dtype in ("fp32", "fp16", "bf16"):
        for d in (-21.0, -24.5, -27.25, -28.5, -30.0, -30.25):
            for cut in (dict(), dict(top_k=2), dict(top_p=1.0 - 2.0**-24), dict(min_p=1e-14)):
                x = torch.full((1, 40000 if not cut else 900), -100.0, device="cuda").to(TYPES[dtype])
                x[0, 17], x[0, 500] = d, 0.0
                token, logprob = ops.sample(x, torch.zeros(1, device="cuda"), return_logprob=True, **cut)
                if int(token) == 500 and "top_p" in cut:
                    continue  # what top_p leaves out may be all of the first
                assert int(token) == 17
                want = d - np.log1p(np.exp(d))
                assert abs(float(logprob) - want) <= 2.0**-23 * abs(want), (dtype, d, float(logprob))


def test_a_tail_below_the_unit(ops):
    """Tokens of less than 2^-45 of the largest one's weight are not drawn, however many they are; the others' borders move by no
    more than the tail's sum, 2^-27 here."""
    vocab = 1 << 19
    for dtype in ("fp32", "bf16"):
        x = torch.full((1, vocab), -32.0, device="cuda").to(TYPES[dtype])  # 2^-46.2
        x[0, [1000, 77_777, 300_000, 500_001]] = torch.tensor([-30.5, -2.0, 0.0, -0.5], device="cuda").to(TYPES[dtype])  # the first: 2^-44.0
        w = torch.exp(x[0].double())
        upto = torch.cumsum(w, 0) / w.sum()
        u = torch.cat([torch.linspace(0, 1, 300, device="cuda")[1:-1], upto[[77_777, 300_000]].float() + 2.0**-22, upto[[77_777, 300_000]].float() - 2.0**-22])
        want = torch.searchsorted(upto, u.double(), right=True)
        for settings in (dict(), dict(temperature=torch.ones(len(u), device="cuda"), top_k=vocab), dict(min_p=1e-15)):
            assert torch.equal(ops.sample(x.expand(len(u), vocab), u, **settings).long(), want)
        assert ops.sample(x, torch.zeros(1, device="cuda")).tolist() == [1000]
