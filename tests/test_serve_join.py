"""The join of a split item: its statistics share memory with what the next item writes, so it has to end in a barrier."""
import os
import re

import numpy as np
import pytest

import serve_ref as ref

torch = pytest.importorskip("torch")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = os.path.join(ROOT, "paper_2002_12798_b200", "csrc", "serve_attend.cu")


def overlaps(dim, parts):
    """(head whose (m, l) the next item writes, part and head whose statistics lie there) with another warp reading them than
    the one that writes, for heads of `dim` elements: rows of dim + 4 floats with (m, l) behind the elements, against an array
    [parts][8] of pairs at the same place that is read by the threads in turn, dim / 4 of them to a head."""
    found = []
    for row in range(32):
        at = (row * (dim + 4) + dim) * 4
        part, head = at // 64, at % 64 // 8
        readers = {(head * (dim // 4) + i) % 128 // 32 for i in range(dim // 4)}
        if part < parts and readers - {row // 8}:
            found.append((row, part, head))
    return found


def test_a_join_ends_in_a_barrier():
    text = open(SOURCE).read()
    direct, group = (int(re.search(r"constexpr int %s = (\d+);" % n, text).group(1)) for n in ("kDirect", "kGroup"))
    assert "kPitch = DP + 4;" in text and "reinterpret_cast<float2(*)[8]>(joint)" in text  # the layout that `overlaps` goes by
    groups = -(-2 * 148 // group)
    assert overlaps(64, direct) and overlaps(128, groups) and overlaps(256, groups)
    body = re.search(r"__device__ void join\(.*?\n}\n", text, re.S).group(0)
    assert body.rstrip("}\n ").splitlines()[-1].strip() == "T::sync();"


@pytest.mark.gpu
@pytest.mark.parametrize("dim,heads,long,parts", [(64, 1, 20, 10), (128, 1, 1, 200)])
def test_short_requests_behind_joined_ones(dim, heads, long, parts):
    """Long requests that about `parts` teams share, each with short ones behind it that the same blocks take up."""
    from paper_2002_12798_b200 import ops

    r = np.random.default_rng(dim)
    torch.manual_seed(dim)
    page, short = 64, 1500
    n_short = short // long
    # a piece of the line, of which there are 296: the short requests' places (3 each) in what the long ones leave over
    piece = 3 * short // (296 - long * parts)
    tokens = parts * piece * (128 if dim == 64 else 64)
    lens = ([tokens - 5] + r.integers(1, 60, n_short).tolist()) * long
    lens = np.array(lens, dtype=np.int32)
    row = -(-tokens // page)
    table = r.permutation(row).astype(np.int32)[None].repeat(len(lens), 0)  # all requests over the same pages
    for i in range(len(lens)):
        table[i] = np.roll(table[i], i)
    k = torch.randn(row, page, heads, dim, device="cuda", dtype=torch.bfloat16)
    v = torch.randn(row, page, heads, dim, device="cuda", dtype=torch.bfloat16)
    q = torch.randn(len(lens), 8 * heads, dim, device="cuda", dtype=torch.bfloat16)
    plan, cache = ops.AttendPlan(len(lens), 8 * heads, heads, dim), ops.PagedCache(k, v)
    args = q, cache, torch.from_numpy(table).cuda(), torch.from_numpy(lens).cuda()
    out, lse = plan.attend(*args, return_lse=True)
    for _ in range(60):
        again, lse_again = plan.attend(*args, return_lse=True)
        assert torch.equal(again, out) and torch.equal(lse_again, lse)
    some = np.concatenate([np.arange(0, len(lens), (n_short + 1) * max(1, long // 4)), np.arange(1, len(lens), 7)])
    some = some[np.argsort(lens[some])[-200:]] if len(some) > 200 else some
    f64 = lambda t: t.float().cpu().double().numpy()  # noqa: E731
    want, want_lse, size, mass = ref.attend(f64(q)[some], f64(k), f64(v), table[some], lens[some], plan.scale)
    bound, lse_bound = ref.attend_bound(want, size, mass, dim, "bf16")
    assert (np.abs(f64(out)[some] - want) <= bound).all()
    assert (np.abs(f64(lse)[some] - want_lse) <= lse_bound + 2.0**-22 * np.abs(want_lse)).all()


def test_a_warp_that_gave_up_waits_for_the_last_copies():
    """`settle` on a model of the ring's barriers: for every number of fills it waits for each stage's last, and for no phase
    that nothing will complete."""
    text = open(SOURCE).read()
    assert "bar_wait_slow(full + 8 * s, s < stage ? parity : parity ^ 1, failed)" in text
    for name, wait in (("consumer", "settle(smem_at(&small.full[0]), S, stage, parity, P.failed)"), ("producer", "settle(smem_at(&small.full[0]), S, stage, parity ^ 1, P.failed)")):
        assert wait in text, name
    assert text.count("if (++stage == S) stage = 0, parity ^= 1;") == 3  # a consumer's step, and the producer's in its two forms
    for stages in (2, 3, 6):
        for fills in range(4 * stages + 1):
            stage, parity = 0, 0  # as a consumer counts; the producer's parity is the other one throughout
            phases = [0] * stages  # completed, once every copy has landed
            for _ in range(fills):
                phases[stage] += 1
                stage += 1
                if stage == stages:
                    stage, parity = 0, parity ^ 1
            for s in range(stages):
                waits_for = parity if s < stage else parity ^ 1
                # a wait for a parity is over when the phase at work has the other one; one copy fewer must not be enough
                over = lambda completed: completed % 2 != waits_for  # noqa: E731
                assert over(phases[s])
                assert phases[s] == 0 or not over(phases[s] - 1)
