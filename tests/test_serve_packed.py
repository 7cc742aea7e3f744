"""The cache of 4 bits without a GPU: where things lie in a cell, and what the operators on it and sampling refuse."""
import ctypes
import os
import re
import shutil
import struct
import subprocess

import numpy as np
import pytest
import torch

import packed_ref as ref
from paper_2002_12798_b200 import binding as B
from paper_2002_12798_b200 import ops

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2002_12798_b200", "csrc")
OK, EINVAL, EOVERFLOW, EALIGN, EUNSUPPORTED = 0, -1, -6, -7, -9
SHAPES = [(64, 32), (64, 64), (96, 32), (128, 32), (128, 64), (256, 32), (256, 64)]

PACKED = struct.Struct("P2q6i")
APPEND, READ, SAMPLE = struct.Struct("q2i4P8qP2q2iP"), struct.Struct("q2i3P4q"), struct.Struct("4iPq5Pfi2f2P")
ATTEND = struct.Struct("4i3P5qPqP2f2iPqP")  # up to its cache, which is not looked at
lib = ctypes.CDLL(B.LIBRARY_PATH)
lib.amap_serve_error.restype = ctypes.c_char_p
lib.amap_packed_bytes.restype = ctypes.c_int64
lib.amap_packed_append.argtypes = [ctypes.c_void_p, ctypes.c_char_p, ctypes.c_void_p]
lib.amap_packed_attend.argtypes = [ctypes.c_char_p, ctypes.c_char_p, ctypes.c_void_p]
for _name in ("amap_packed_read", "amap_sample"):
    getattr(lib, _name).argtypes = [ctypes.c_char_p, ctypes.c_void_p]


def test_structs_are_as_long_as_the_header_says(tmp_path):
    cc = shutil.which("gcc")
    if not cc:
        pytest.skip("no C compiler")
    sizes = {"amap_packed": PACKED.size, "amap_packed_append_args": APPEND.size + PACKED.size, "amap_packed_read_args": READ.size + PACKED.size,
             "amap_sample_args": SAMPLE.size}
    assert ctypes.sizeof(ops._Packed) == PACKED.size
    src = tmp_path / "sizes.c"
    src.write_text('#include "amap_serve.h"\n' + "".join('_Static_assert(sizeof(%s) == %d, "%s");\n' % (n, s, n) for n, s in sizes.items())
                   + "int main(void) { return 0; }\n")
    subprocess.check_call([cc, "-std=c11", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), "-c", str(src), "-o", str(tmp_path / "sizes.o")])


@pytest.fixture(scope="module")
def places(tmp_path_factory):
    """For every shape, the offsets of everything that belongs to each token of a cell."""
    cxx = shutil.which("g++")
    if not cxx:
        pytest.skip("no C++ compiler")
    d = tmp_path_factory.mktemp("places")
    (d / "places.cpp").write_text("""
#include <cstdio>
#include "serve_packed.cuh"
using namespace amap_serve;
int main() {
  const int shapes[7][2] = {%s};
  for (auto &s : shapes) {
    const int slabs = s[0] / 32, groups = s[0] / s[1];
    printf("shape %%d %%d %%d\\n", s[0], s[1], cell_bytes(slabs, groups));
    for (int t = 0; t < 16; ++t) {
      for (int c = 0; c < s[0] / 8; ++c) printf("k %%d %%d %%d\\n", t, c, k_word_at(slabs, t, c));
      for (int f = 0; f < s[0] / 4; ++f) printf("v %%d %%d %%d\\n", t, f, v_half_at(slabs, t, f));
      for (int g = 0; g < groups; ++g) printf("n %%d %%d %%d\\n", t, g, numbers_at(slabs, t, g));
    }
  }
}
""" % ", ".join("{%d, %d}" % s for s in SHAPES))
    flags = ["-std=c++17", "-O1", "-Wall", "-Werror", "-I", CSRC, "-I", os.path.join(ROOT, "include"), "-x", "c++"]
    subprocess.check_call([cxx, *flags, str(d / "places.cpp"), "-o", str(d / "places")])
    found, at = {}, None
    for line in subprocess.check_output([str(d / "places")], text=True).splitlines():
        kind, a, b, c = line.split()
        if kind == "shape":
            at = found[int(a), int(b)] = {"bytes": int(c), "k": {}, "v": {}, "n": {}}
        else:
            at[kind][int(a), int(b)] = int(c)
    return found


@pytest.mark.parametrize("dim,group", SHAPES)
def test_a_cell_is_tiled_by_its_tokens(places, dim, group):
    p = places[dim, group]
    owner = np.full(p["bytes"], -1)
    for kind, size in (("k", 4), ("v", 2), ("n", 4)):
        for (token, _), at in p[kind].items():
            for first in (at, at + 4) if kind == "n" else (at,):  # V's numbers lie behind K's
                assert at % size == 0 and (owner[first : first + size] == -1).all()
                owner[first : first + size] = token
    assert (owner >= 0).all() and p["bytes"] % 128 == 0
    assert lib.amap_packed_bytes(48, dim, group) == 3 * p["bytes"]


@pytest.mark.parametrize("dim,group", SHAPES)
def test_lanes_find_their_operands(places, dim, group):
    """The addresses that attention's lanes load from (serve_attend_packed.cu), against where the writers put things."""
    p, slabs = places[dim, group], dim // 32
    for lane in range(32):
        g, t4 = lane >> 2, lane & 3
        for slab in range(slabs):
            first = slab // 4 * 4
            wide = min(4, slabs - first)
            for token in (g, g + 8):
                assert p["k"][token, 4 * slab + t4] == first * 256 + (token * 4 + t4) * 4 * wide + (slab - first) * 4
            first = slab // 2 * 2
            wide = min(2, slabs - first)
            for token in range(16):
                if (token & 7) >> 1 == t4:
                    word = slabs * 256 + first * 256 + lane * 8 * wide + (slab - first) * 8 + (token >> 3) * 4
                    assert p["v"][token, 8 * slab + g] == word + 2 * (token & 1)
        for n in range(dim // group):
            for e in range(2):
                assert p["n"][8 * e + g, n] == slabs * 512 + g * 8 + n * 128 + e * 64


def test_the_reference_quantises_as_defined():
    r = np.random.default_rng(0)
    x = r.standard_normal((50, 128)) * np.exp(3 * r.standard_normal((50, 1)))
    codes, low, step = ref.quantise(x, 32)
    g = x.reshape(50, 4, 32)
    assert (low <= g.min(-1)).all() and (low + np.abs(low) * 2.0**-7 >= g.min(-1)).all()
    assert set(np.unique(codes)) <= set(range(16)) and (codes.reshape(50, 4, 32).min(-1) == 0).any()
    # half a step, and what the step's rounding leaves at the top (15 of 2^-9 of it)
    assert (np.abs(ref.held(x, 32).reshape(50, 4, 32) - g) <= step[..., None] * (0.5 + 15 * 2.0**-9)).all()
    for b in (low, step):
        assert (b == torch.from_numpy(b).to(torch.bfloat16).double().numpy()).all()


# ----------------------------------------------------------------------------------------------------------------------
# refusals
# ----------------------------------------------------------------------------------------------------------------------
def refused(rc, code, why):
    text = lib.amap_serve_error().decode()
    assert rc == code and why in text, (rc, text)


CACHE = dict(data=0x100000, page=8 * 2304, head=2304, pages=4, page_size=16, heads=8, dim=128, group=64, reserved=0)
CACHE_REFUSALS = [
    (dict(data=0), EINVAL, "null"), (dict(pages=0), EINVAL, "at least 1"), (dict(heads=0), EINVAL, "at least 1"), (dict(reserved=1), EINVAL, "at least 1"),
    (dict(page_size=8), EUNSUPPORTED, "multiple of 16"), (dict(page_size=0), EUNSUPPORTED, "multiple of 16"), (dict(page_size=24), EUNSUPPORTED, "multiple of 16"),
    (dict(dim=80), EUNSUPPORTED, "64, 96, 128 or 256"), (dict(group=128), EUNSUPPORTED, "groups"), (dict(dim=96), EUNSUPPORTED, "groups"),
    (dict(pages=2**27), EOVERFLOW, "2^31"), (dict(data=0x100008), EALIGN, "16 bytes"), (dict(page=8 * 2304 + 8), EALIGN, "16 bytes"),
    (dict(head=2288), EINVAL, "overlap"), (dict(page=7 * 2304), EINVAL, "overlap"), (dict(page=0), EINVAL, "overlap"), (dict(head=-16), EINVAL, "overlap"),
    (dict(page=2**62), EOVERFLOW, "beyond"), (dict(head=-2**62), EOVERFLOW, "beyond"),
]


def cache_of(change):
    return PACKED.pack(*{**CACHE, **change}.values())


READ_ARGS = dict(rows=5, dtype=1, reserved=0, slots=0x1000, k=0x200000, v=0x300000, k_row=1024, k_head=128, v_row=1024, v_head=128)


def read(change, cache=None):
    return lib.amap_packed_read(READ.pack(*{**READ_ARGS, **change}.values()) + cache_of(cache or {}), None)


@pytest.mark.parametrize("change,code,why", CACHE_REFUSALS)
def test_caches(change, code, why):
    refused(read({}, change), code, why)
    refused(append({}, change), code, why)
    refused(attend({}, change), code, why)


@pytest.mark.parametrize("change,code,why", [
    (dict(dtype=4), EINVAL, "type"), (dict(rows=-1), EINVAL, "rows"), (dict(reserved=1), EINVAL, "rows"), (dict(slots=0), EINVAL, "null"),
    (dict(k=0), EINVAL, "null"), (dict(k=0x200001), EALIGN, "misaligned"), (dict(slots=0x1002), EALIGN, "misaligned"), (dict(k_row=0), EINVAL, "on one another"),
    (dict(v_head=0), EINVAL, "on one another"), (dict(v=0x200100), EINVAL, "share"), (dict(k=0x100000), EINVAL, "overlaps the cache"),
])
def test_read(change, code, why):
    refused(read(change), code, why)


def test_no_rows_are_read():
    assert read(dict(rows=0, k=0)) == OK


def test_page_strides_either_way():
    """Heads outside pages, and pages outside heads: neither overlaps (the calls get as far as their null pointers)."""
    refused(read(dict(k=0), dict(page=2304, head=4 * 2304)), EINVAL, "null pointer")
    refused(read(dict(k=0), dict(page=-8 * 2304, head=2304)), EINVAL, "null pointer")
    refused(read(dict(k=0), dict(page=2304, head=3 * 2304)), EINVAL, "overlap")


APPEND_ARGS = dict(rows=5, dtype=1, q_heads=32, q=0x400000, k=0x500000, v=0x600000, out=0x700000, q_row=4096, q_head=128, k_row=1024, k_head=128,
                   v_row=1024, v_head=128, out_row=4096, out_head=128, pos=0x2000, axis=0, row=1, bits=32, reserved=0, slots=0x1000)


def append(change, cache=None, plan=True):
    made = ops.RopePlan(128 if "dim" not in change else change.pop("dim"))
    return lib.amap_packed_append(made._h if plan else None, APPEND.pack(*{**APPEND_ARGS, **change}.values()) + cache_of(cache or {}), None)


@pytest.mark.parametrize("change,code,why", [
    (dict(dtype=3), EINVAL, "type"), (dict(rows=-1), EINVAL, "rows"), (dict(bits=16), EINVAL, "32 or 64"), (dict(pos=0), EINVAL, "null"),
    (dict(pos=0x2002), EALIGN, "misaligned"), (dict(dim=64), EINVAL, "differs"), (dict(q_heads=-1), EINVAL, "65535"), (dict(reserved=1), EINVAL, "65535"),
    (dict(k=0), EINVAL, "null"), (dict(out=0), EINVAL, "null"), (dict(slots=0x1001), EALIGN, "misaligned"), (dict(v=0x600001), EALIGN, "misaligned"),
    (dict(out_row=0), EINVAL, "on one another"), (dict(out=0x400080), EINVAL, "overlaps"), (dict(out=0x500000), EINVAL, "overlaps"),
    (dict(out=0x100000), EINVAL, "overlaps the cache"), (dict(k=0x100000), EINVAL, "overlaps the cache"),
])
def test_append(change, code, why):
    refused(append(dict(change)), code, why)


def test_append_without_a_plan_reads_no_positions():
    refused(append(dict(pos=0, bits=0, v=0), plan=False), EINVAL, "null pointer")
    assert append(dict(rows=0, pos=0, bits=0, v=0), plan=False) == OK


ATTEND_ARGS = dict(n=4, q_heads=32, dtype=1, max_pages=8, q=0x400000, out=0x500000, lse=0, q_row=4096, q_head=128, out_row=4096, out_head=128, lse_row=32,
                   table=0x3000, table_stride=8, lens=0x4000, scale=0.1, softcap=0.0, window=0, reserved=0, workspace=0x800000, bytes=1 << 40, maps=0)


def attend(change, cache=None):
    return lib.amap_packed_attend(ATTEND.pack(*{**ATTEND_ARGS, **change}.values()) + bytes(128), cache_of(cache or {}), None)


@pytest.mark.parametrize("change,code,why", [
    (dict(n=0), EINVAL, "65535"), (dict(q_heads=30), EINVAL, "multiple"), (dict(dtype=4), EINVAL, "bf16 or fp16"), (dict(q=0), EINVAL, "null"),
    (dict(workspace=0x800010), EALIGN, "misaligned"), (dict(table_stride=7), EINVAL, "overlap"), (dict(max_pages=2**27, table_stride=2**27), EOVERFLOW, "2^31"),
    (dict(scale=float("nan")), EINVAL, "finite"), (dict(window=-1), EINVAL, "negative"), (dict(out=0x400000), EINVAL, "overlap"), (dict(bytes=1000), EINVAL, "too small"),
])
def test_attend(change, code, why):
    refused(attend(change), code, why)


SAMPLE_ARGS = dict(rows=4, vocab=1000, dtype=1, by_row=0, logits=0x10000, row=1000, uniform=0x20000, temps=0, ks=0, ps=0, ms=0, t=1.0, k=0, p=1.0, m=0.0,
                   tokens=0x30000, logprobs=0)


@pytest.mark.parametrize("change,code,why", [
    (dict(rows=0), EINVAL, "rows"), (dict(rows=65536), EINVAL, "rows"), (dict(vocab=0), EINVAL, "vocab"), (dict(vocab=2**19 + 1), EINVAL, "vocab"),
    (dict(dtype=4), EINVAL, "type"), (dict(by_row=16), EINVAL, "by_row"), (dict(by_row=1), EINVAL, "null"), (dict(by_row=2), EINVAL, "null"),
    (dict(by_row=4), EINVAL, "null"), (dict(by_row=8), EINVAL, "null"), (dict(logits=0), EINVAL, "null"), (dict(uniform=0), EINVAL, "null"),
    (dict(tokens=0), EINVAL, "null"), (dict(t=float("nan")), EINVAL, "temperature"), (dict(t=float("inf")), EINVAL, "temperature"), (dict(p=1.5), EINVAL, "top_p"),
    (dict(p=-0.1), EINVAL, "top_p"), (dict(p=float("nan")), EINVAL, "top_p"), (dict(m=1.1), EINVAL, "min_p"), (dict(logits=0x10001), EALIGN, "misaligned"),
    (dict(tokens=0x30002), EALIGN, "misaligned"), (dict(logprobs=0x30002), EALIGN, "misaligned"),
])
def test_sample(change, code, why):
    refused(lib.amap_sample(SAMPLE.pack(*{**SAMPLE_ARGS, **change}.values()), None), code, why)


def test_python_refusals():
    x = torch.zeros(2, 10)
    with pytest.raises(ValueError, match="CPU"):
        ops.sample(x, torch.zeros(2))
    with pytest.raises(ValueError, match="not a tensor"):
        ops.sample([1.0], torch.zeros(1))
    with pytest.raises(ValueError, match="multiple of 16"):
        ops.PackedCache.page_bytes(24, 128)
    with pytest.raises(ValueError, match="uint8 CUDA tensor"):
        ops.PackedCache(torch.zeros(4, 8, ops.PackedCache.page_bytes(16, 128), dtype=torch.uint8), 16, 128)
    assert ops.PackedCache.page_bytes(16, 128) == 2304 and ops.PackedCache.page_bytes(32, 128, 32) == 5120


def test_the_kernel_and_the_layout_name_the_same_cell():
    text = open(os.path.join(CSRC, "serve_packed.cuh")).read()
    assert int(re.search(r"constexpr int kCell = (\d+);", text).group(1)) == 16


def test_codes_lie_where_the_masks_find_them(tmp_path):
    """The two masks of attention (serve_attend_packed.cu) on a word, and on it with its halves' bytes exchanged, give all eight codes."""
    cxx = shutil.which("g++")
    if not cxx:
        pytest.skip("no C++ compiler")
    (tmp_path / "codes.cpp").write_text("""
#include <cstdio>
#include "serve_packed.cuh"
int main() {
  for (uint32_t i = 0, w = 0x12345678u; i < 200; ++i, w = w * 1664525u + 1013904223u)
    printf("%u %u\\n", w, amap_serve::turn_halves(w));
}
""")
    flags = ["-std=c++17", "-O1", "-Wall", "-Werror", "-I", CSRC, "-I", os.path.join(ROOT, "include"), "-x", "c++"]
    subprocess.check_call([cxx, *flags, str(tmp_path / "codes.cpp"), "-o", str(tmp_path / "codes")])
    text = open(os.path.join(CSRC, "serve_attend_packed.cu")).read()
    lower, upper = (int(x, 16) for x in re.search(r"kLower = (0x\w+)u, kUpper = (0x\w+)u;", text).groups())
    for line in subprocess.check_output([str(tmp_path / "codes")], text=True).splitlines():
        plain, held = (int(x) for x in line.split())
        other = (held & 0x00FF00FF) << 8 | held >> 8 & 0x00FF00FF
        got = [(x & mask) >> shift >> 16 * o & 0xFFFF for x in (held, other) for mask, shift in ((lower, 3), (upper, 7)) for o in (0, 1)]
        assert got == [plain >> (4 * i + 16 * o) & 15 for i in range(4) for o in (0, 1)]
