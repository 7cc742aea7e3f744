"""Decode attention at the longest lengths that it accepts: one token's memory stands for all of a page's (stride 0), and a
window leaves the last few."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("page,pages", [(2**31 - 1, 1), (2**30 - 1, 2), (2**31 - 8, 1)])
@pytest.mark.parametrize("window", [1, 100, 200, 1000])
def test_attend_lengths_up_to_31_bits(dim, page, pages, window):
    from paper_2002_12798_b200 import ops

    k = torch.randn(1, 1, 2, dim, device="cuda", dtype=torch.bfloat16)
    v = torch.randn(1, 1, 2, dim, device="cuda", dtype=torch.bfloat16)
    cache = ops.PagedCache(k.expand(1, page, 2, dim), v.expand(1, page, 2, dim))
    room = page * pages
    lens = np.array([room, room - 1, room - 62, 5, room - 130, 2**31 - 1], dtype=np.int64).clip(max=2**31 - 1).astype(np.int32)
    table = torch.zeros(len(lens), pages, dtype=torch.int32, device="cuda")
    q = torch.randn(len(lens), 4, dim, device="cuda", dtype=torch.bfloat16)
    out, lse = ops.AttendPlan(len(lens), 4, 2, dim, window=window).attend(q, cache, table, torch.from_numpy(lens).cuda(), return_lse=True)
    score = torch.einsum("rhgd,hd->rhg", q.double().view(-1, 2, 2, dim), k[0, 0].double()).reshape(-1, 4) / math.sqrt(dim)
    count = torch.tensor([min(int(n), room, window) for n in lens], dtype=torch.float64, device="cuda")
    # a score's dim products in 32 bits, at most 2^-23 dim of the sum of their sizes
    size = torch.einsum("rhgd,hd->rhg", q.double().abs().view(-1, 2, 2, dim), k[0, 0].double().abs()).reshape(-1, 4)
    assert ((lse.double() - (score + count.log()[:, None])).abs() <= 2.0**-14 + (dim + 16) * 2.0**-23 * size).all()
    assert (out.double() - v[0, 0].double().repeat_interleave(2, 0)).abs().max() <= 2.0**-7 * v.abs().max()
