"""Pages given back from table rows with holes."""
import ctypes

import numpy as np
import pytest

import test_serve_refusals as T

torch = pytest.importorskip("torch")


def test_release_within_refuses():
    lib = T.lib
    lib.amap_pages_release_within.argtypes = [ctypes.c_char_p, ctypes.c_int32, ctypes.c_void_p]
    T.refused(lib.amap_pages_release_within(T.RELEASE_ARGS.pack(*T.RELEASE.values()), 0, None), T.EINVAL, "pages")
    T.refused(lib.amap_pages_release_within(T.RELEASE_ARGS.pack(*{**T.RELEASE, "done": 0}.values()), 64, None), T.EINVAL, "null")


def by_definition(done, seq, table, free, count, page, n_pages):
    free, out = free.copy(), seq.copy()
    for r in np.nonzero(done)[0]:
        length = min(max(int(seq[r]), 0), table.shape[1] * page)
        for e in table[r, : -(-length // page)].tolist():
            if 0 <= e < n_pages and count < len(free):
                free[count] = e
                count += 1
        out[r] = 0
    return out, count, free


@pytest.mark.gpu
@pytest.mark.parametrize("requests,row", [(1, 1), (3, 40), (9, 300), (64, 33), (1000, 31), (1024, 40), (1025, 600), (5000, 12)])
@pytest.mark.parametrize("holes", [0.0, 0.1, 1.0])
@pytest.mark.parametrize("limit", [False, True])
def test_release_passes_over_holes(requests, row, holes, limit):
    from paper_2002_12798_b200 import ops

    r = np.random.default_rng(requests + row)
    page, spare = 16, 7
    seq = r.integers(-1, row * page + 40, requests).astype(np.int32)
    done = r.random(requests) < 0.5
    total = requests * row
    table = r.permutation(total).astype(np.int32).reshape(requests, row)
    at = r.random((requests, row)) < holes
    table[at] = r.choice([-1, -(2**31), -7], at.sum()) if not limit else r.choice([-1, total, 2**31 - 1, -5], at.sum())
    for capacity in (total + spare, max(spare, total // 3)):
        free = np.full(capacity, -9, dtype=np.int32)
        free[:spare] = total + np.arange(spare)
        want = by_definition(done, seq, table, free, spare, page, total if limit else 2**31)
        wide = torch.from_numpy(np.pad(table, ((0, 0), (0, 3)), constant_values=5)).cuda()
        got = torch.from_numpy(free).cuda()
        seq_out, count = ops.pages_release(torch.from_numpy(done).cuda(), torch.from_numpy(seq).cuda(), wide[:, :row], got,
                                           torch.tensor([spare], dtype=torch.int32).cuda(), page, n_pages=total if limit else None)
        assert np.array_equal(seq_out.cpu().numpy(), want[0]) and int(count) == want[1]
        assert np.array_equal(got.cpu().numpy(), want[2])


@pytest.mark.gpu
def test_pages_behind_a_window_given_back_early():
    """A caller frees the pages behind a window itself and marks them; releasing the request later gives back the rest, and
    the next request gets real pages."""
    from paper_2002_12798_b200 import ops

    one = dict(dtype=torch.int32, device="cuda")
    table, free, count = torch.full((2, 8), -1, **one), torch.arange(8, **one), torch.tensor([8], **one)
    step = ops.pages_extend(torch.tensor([30, 0], **one), torch.zeros(2, **one), table, free, count, 4, 30)
    assert step.status.tolist() == [0, 0] and int(step.free_count) == 0
    free[0], free[1] = table[0, 0].clone(), table[0, 1].clone()
    table[0, :2] = -1
    seq, count = ops.pages_release(torch.tensor([True, False], device="cuda"), step.seq_lens, table, free, torch.tensor([2], **one), 4)
    assert int(count) == 8 and sorted(free.tolist()) == list(range(8))
    step = ops.pages_extend(torch.tensor([0, 32], **one), seq, table, free, count, 4, 32)
    assert step.status.tolist() == [0, 0] and (step.slots >= 0).all() and len(set(step.slots.tolist())) == 32
