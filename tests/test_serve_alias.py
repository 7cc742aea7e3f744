"""Parts of one call that share memory: what the check of strided tensors says, and what rotate and append refuse."""
import os
import shutil
import subprocess

import pytest
import torch

import test_serve_refusals as T
from paper_2002_12798_b200 import ops

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <cstdio>
#include <random>
#include <vector>
#include "serve_alias.hpp"
using namespace amap_serve;
int main() {
  std::mt19937 r(5);
  auto pick = [&](int lo, int hi) { return (int64_t)std::uniform_int_distribution<int>(lo, hi)(r); };
  long shared = 0, apart = 0, careful = 0;
  for (int t = 0; t < 400000; ++t) {
    const int64_t width = pick(1, 5);
    Runs a = {200 + pick(-40, 40), pick(1, 5), pick(-30, 30), pick(1, 4), pick(-12, 12)}, b = {200 + pick(-40, 40), pick(1, 5), pick(-30, 30), pick(1, 4), pick(-12, 12)};
    if (pick(0, 3)) b.row = a.row;
    if (pick(0, 1)) b.head = a.head;
    std::vector<char> at(1000);
    for (int64_t i = 0; i < a.rows; ++i) for (int64_t j = 0; j < a.heads; ++j) for (int64_t w = 0; w < width; ++w) at[a.at + i * a.row + j * a.head + w + 100] = 1;
    bool want = false;
    for (int64_t i = 0; i < b.rows; ++i) for (int64_t j = 0; j < b.heads; ++j) for (int64_t w = 0; w < width; ++w) want |= at[b.at + i * b.row + j * b.head + w + 100];
    const bool got = share(a, b, width), exact = a.rows == 1 || b.rows == 1 || a.row == b.row;
    if (exact ? got != want : want && !got) {
      printf("wrong: %d for %ld (%ld x %ld, %ld x %ld), %ld (%ld x %ld, %ld x %ld), width %ld\n", got, a.at, a.rows, a.row, a.heads, a.head, b.at, b.rows, b.row, b.heads, b.head, width);
      return 1;
    }
    ++(want ? shared : got ? careful : apart);
  }
  printf("%ld %ld %ld\n", shared, apart, careful);
  return shared > 50000 && apart > 50000 ? 0 : 1;
}
"""


def test_share_against_every_byte(tmp_path):
    cxx = shutil.which("g++")
    if not cxx:
        pytest.skip("no C++ compiler")
    (tmp_path / "share.cpp").write_text(PROGRAM)
    flags = ["-std=c++17", "-O2", "-Wall", "-fsanitize=undefined,address", "-I", os.path.join(ROOT, "paper_2002_12798_b200", "csrc")]
    subprocess.check_call([cxx, *flags, str(tmp_path / "share.cpp"), "-o", str(tmp_path / "share")])
    said = subprocess.run([str(tmp_path / "share")], capture_output=True, text=True)
    assert said.returncode == 0, said.stdout + said.stderr


def test_rotate_refuses_parts_that_share_memory():
    plan = ops.RopePlan(64)
    whole = (256, 64, 256, 64, 4, 0)  # 8 rows of 4 heads
    q, k, y = 0x10000, 0x20000, 0x30000
    T.refused(T.rotate(plan, [(q, q) + whole, (q, y) + whole]), T.EINVAL, "share")  # one part in place, read by the other
    T.refused(T.rotate(plan, [(q, y) + whole, (q, q) + whole]), T.EINVAL, "share")
    T.refused(T.rotate(plan, [(q, y) + whole, (k, y) + whole]), T.EINVAL, "share")  # two into one
    T.refused(T.rotate(plan, [(q, q) + whole, (q, q) + whole]), T.EINVAL, "share")  # twice in place
    T.refused(T.rotate(plan, [(q, y) + whole, (k, y + 2 * 63) + whole]), T.EINVAL, "share")  # the last element of the first
    # 8 rows of 6 heads in one buffer: the first 4 and the last 3 heads have one in common
    T.refused(T.rotate(plan, [(q, q, 384, 64, 384, 64, 4, 0), (q + 2 * 3 * 64, q + 2 * 3 * 64, 384, 64, 384, 64, 3, 0)]), T.EINVAL, "share")
    # in place, of overlapping bytes, with other rows
    T.refused(T.rotate(plan, [(q, q) + whole, (q + 512, q + 512, 384, 64, 384, 64, 1, 0)]), T.EINVAL, "share")


def test_append_refuses_a_q_in_place_that_shares_memory_with_k_or_v():
    plan = ops.RopePlan(64)
    for change in (dict(k=0x1000, kr=512), dict(v=0x1000 + 2 * 7 * 64, vr=512), dict(k=0x1000 + 2 * 5 * 64, kr=512)):
        a, c = T.split({**change, "out": 0x1000}, T.APPEND)
        T.refused(T.lib.amap_rope_append(plan._h, T.APPEND_ARGS.pack(*a.values()) + T.CACHE_ARGS.pack(*c.values()), None), T.EINVAL, "overlaps")


@pytest.mark.gpu
def test_parts_in_place_side_by_side():
    """Views of one buffer without a common element are turned as if they were apart: heads side by side, every other head,
    every other row, heads before rows."""
    plan = ops.RopePlan(64)
    pos = torch.arange(6, dtype=torch.int32, device="cuda")
    x = torch.randn(12, 8, 64, device="cuda")
    by_head = torch.randn(8, 6, 64, device="cuda").transpose(0, 1)
    for views in ([x[:6, :3], x[:6, 3:4], x[:6, 4:]], [x[:6, 0::2], x[:6, 1::2]], [x[0::2], x[1::2]], [by_head[:, :5], by_head[:, 5:]],
                  [x[0:6, ::3], x[0:6, 1:3], x[6:, :]]):
        want = plan.rotate(views, pos)
        plan.rotate(views, pos, outs=views)
        assert all(torch.equal(v, w) for v, w in zip(views, want))
    fused = torch.randn(6, 12, 64, device="cuda", dtype=torch.bfloat16)
    cache = ops.PagedCache(*(torch.zeros(1, 8, 2, 64, device="cuda", dtype=torch.bfloat16) for _ in range(2)))
    q, k, v = fused[:, :8], fused[:, 8:10], fused[:, 10:]
    want = plan.append(q, k, v, pos, pos, cache)
    assert plan.append(q, k, v, pos, pos, cache, out=q).data_ptr() == q.data_ptr() and torch.equal(q, want)
    with pytest.raises(Exception, match="share"):
        plan.rotate([q, q], pos, outs=[q, torch.empty_like(q)])
