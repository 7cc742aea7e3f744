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
