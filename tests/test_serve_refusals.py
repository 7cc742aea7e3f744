"""What the serving operators refuse, before anything is enqueued: no GPU is needed to be told so.  Pointers here are
numbers that no call gets as far as using."""
import ctypes
import os
import re
import struct

import pytest
import torch

from paper_2002_12798_b200 import binding as B
from paper_2002_12798_b200 import ops

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, EINVAL, EOVERFLOW, EALIGN, EUNSUPPORTED = 0, -1, -6, -7, -9

# the argument structs of amap_serve.h, with C's alignment
EXTEND_ARGS, RELEASE_ARGS = struct.Struct("6iq12P"), struct.Struct("4iq7P")
ROTATE_ARGS, PART_ARGS = struct.Struct("2iqP2q2i"), struct.Struct("2P4q2i")  # up to part[], and one of part[]
APPEND_ARGS, ATTEND_ARGS = struct.Struct("q2i4P8qP2q2iP"), struct.Struct("4i3P5qPqP2f2iPqP")  # up to cache
CACHE_ARGS, MAPS_ARGS = struct.Struct("2P6q4ii2f4x"), struct.Struct("32Q2i")

lib = ctypes.CDLL(B.LIBRARY_PATH)
lib.amap_serve_error.restype = ctypes.c_char_p
for _name in ("amap_pages_extend", "amap_pages_release", "amap_cache_encode", "amap_attend"):
    getattr(lib, _name).argtypes = [ctypes.c_char_p, ctypes.c_void_p]
for _name in ("amap_rope_rotate", "amap_rope_append"):
    getattr(lib, _name).argtypes = [ctypes.c_void_p, ctypes.c_char_p, ctypes.c_void_p]


def test_library_exports_every_declared_symbol():
    header = open(os.path.join(ROOT, "include", "amap_serve.h")).read()
    header = re.sub(r"/\*.*?\*/", "", header, flags=re.S)
    declared = set(re.findall(r"\b(amap_[a-z_]+)\s*\(", header))
    assert declared == set(ops.EXPORTS)
    for name in declared:
        assert hasattr(ctypes.CDLL(B.LIBRARY_PATH), name), name


def test_packed_structs_are_as_long_as_the_header_says(tmp_path):
    import shutil
    import subprocess

    cc = shutil.which("gcc")
    if not cc:
        pytest.skip("no C compiler")
    sizes = {"amap_pages_extend_args": EXTEND_ARGS.size, "amap_pages_release_args": RELEASE_ARGS.size,
             "amap_rope_args": ROTATE_ARGS.size + 4 * PART_ARGS.size, "amap_rope_part": PART_ARGS.size,
             "amap_append_args": APPEND_ARGS.size + CACHE_ARGS.size, "amap_attend_args": ATTEND_ARGS.size + CACHE_ARGS.size,
             "amap_cache": CACHE_ARGS.size, "amap_cache_maps": MAPS_ARGS.size}
    checks = "".join("_Static_assert(sizeof(%s) == %d, \"%s\");\n" % (n, s, n) for n, s in sizes.items())
    assert sizes["amap_cache"] == ctypes.sizeof(ops._Cache) and sizes["amap_cache_maps"] == ctypes.sizeof(ops._Maps)
    assert sizes["amap_attend_args"] == ctypes.sizeof(ops._Attend)
    src = tmp_path / "sizes.c"
    src.write_text('#include "amap_serve.h"\n' + checks + "int main(void) { return 0; }\n")  # the header is C, too
    subprocess.check_call([cc, "-std=c11", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), "-c", str(src), "-o", str(tmp_path / "sizes.o")])


def refused(rc, code, why):
    text = lib.amap_serve_error().decode()
    assert rc == code and why in text, (rc, text)


EXTEND = dict(n=4, row=8, page=16, pages=64, capacity=64, tokens=100, stride=8, new=0x10000, seq=0x20000, table=0x30000, free=0x40000,
              count=0x50000, start=0x60000, slots=0x70000, pos=0x80000, req=0x90000, seq_out=0xA0000, count_out=0xB0000, status=0xC0000)


@pytest.mark.parametrize("change,code,why", [
    (dict(n=0), EINVAL, "at least 1"), (dict(page=0), EINVAL, "at least 1"), (dict(row=0), EINVAL, "at least 1"), (dict(tokens=0), EINVAL, "at least 1"),
    (dict(capacity=-1), EINVAL, "at least 1"), (dict(stride=7), EINVAL, "overlap"), (dict(row=2**27, stride=2**27), EOVERFLOW, "2^31"),
    (dict(pages=2**27), EOVERFLOW, "2^31"), (dict(slots=0), EINVAL, "null"), (dict(free=0), EINVAL, "null"), (dict(seq=0x20002), EALIGN, "misaligned"),
    (dict(seq_out=0x20000), EINVAL, "overlaps"), (dict(count_out=0x50000), EINVAL, "overlaps"), (dict(slots=0x80004), EINVAL, "overlaps"),
])
def test_extend(change, code, why):
    refused(lib.amap_pages_extend(EXTEND_ARGS.pack(*{**EXTEND, **change}.values()), None), code, why)


RELEASE = dict(n=4, row=8, page=16, capacity=64, stride=8, done=0x10001, seq=0x20000, table=0x30000, free=0x40000, count=0x50000,
               seq_out=0xA0000, count_out=0xB0000)


@pytest.mark.parametrize("change,code,why", [
    (dict(n=-1), EINVAL, "at least 1"), (dict(stride=0), EINVAL, "overlap"), (dict(done=0), EINVAL, "null"), (dict(table=0x30001), EALIGN, "misaligned"),
    (dict(seq_out=0x20004), EINVAL, "overlaps"), (dict(free=0x30010), EINVAL, "overlaps"),
])
def test_release(change, code, why):
    refused(lib.amap_pages_release(RELEASE_ARGS.pack(*{**RELEASE, **change}.values()), None), code, why)


@pytest.mark.parametrize("args,why", [
    (dict(head_dim=0), "head_dim"), (dict(head_dim=257), "head_dim"), (dict(head_dim=64, rotary_dim=66), "rotary_dim"),
    (dict(head_dim=64, rotary_dim=33), "rotary_dim"), (dict(head_dim=64, inv_freq=[float("nan")] * 32), "inv_freq"),
    (dict(head_dim=64, axes=[0] * 31 + [4]), "n_axes"), (dict(head_dim=64, axes=[0] * 31 + [-1]), "axis"), (dict(head_dim=64, scale=float("inf")), "scale"),
])
def test_rope_plan(args, why):
    with pytest.raises(B.AmapError) as e:
        ops.RopePlan(args.pop("head_dim"), args.pop("rotary_dim", None), **args)
    assert e.value.code == EINVAL and why in str(e.value)


@pytest.mark.parametrize("args", [dict(inv_freq=[1.0]), dict(axes=[0]), dict(sections=[1, 2]), dict(sections=[32], axes=[0] * 32), dict(pairs="odd")])
def test_rope_plan_arguments(args):
    with pytest.raises(ValueError):
        ops.RopePlan(64, **args)


def rotate(plan, parts, n=None, dtype=1, rows=8, positions=0x100, axis=8, row=1, bits=32, inverse=0):
    packed = [PART_ARGS.pack(*p) for p in parts]
    head = ROTATE_ARGS.pack(len(parts) if n is None else n, dtype, rows, positions, axis, row, bits, inverse)
    return lib.amap_rope_rotate(plan._h, head + b"".join(packed) + bytes((4 - len(parts)) * PART_ARGS.size), None)


def test_rotate():
    plan = ops.RopePlan(64)
    part = (0x10000, 0x20000, 256, 64, 256, 64, 4, 0)
    refused(rotate(plan, [], n=0), EINVAL, "n_parts")
    refused(rotate(plan, [part], n=5), EINVAL, "n_parts")
    refused(rotate(plan, [part], dtype=4), EINVAL, "type")
    refused(rotate(plan, [part], rows=-1), EINVAL, "rows")
    refused(rotate(plan, [part], bits=16), EINVAL, "positions")
    refused(rotate(plan, [part], positions=0), EINVAL, "positions")
    refused(rotate(plan, [part], positions=0x104, bits=64), EALIGN, "positions")
    refused(rotate(plan, [(0,) + part[1:]]), EINVAL, "null")
    refused(rotate(plan, [part[:6] + (0, 0)]), EINVAL, "heads")
    refused(rotate(plan, [(0x10001,) + part[1:]]), EALIGN, "misaligned")
    refused(rotate(plan, [(0x10000, 0x10002) + part[2:]]), EINVAL, "overlaps")
    refused(rotate(plan, [part, (0x20000, 0x40000) + part[2:]]), EINVAL, "overlaps")  # one part's output is another's input
    refused(rotate(plan, [(0x10000, 0x20000, 256, 64, 256, 0, 4, 0)]), EINVAL, "on one another")
    refused(lib.amap_rope_rotate(None, bytes(ROTATE_ARGS.size + 4 * PART_ARGS.size), None), EINVAL, "null")
    assert rotate(plan, [part], rows=0) == OK  # nothing to do, nothing enqueued


CACHE = dict(k=0x100000, v=0x200000, kp=4096, kt=256, kh=64, vp=4096, vt=256, vh=64, pages=8, page=16, heads=4, dim=64, dtype=1, ks=1.0, vs=1.0)
APPEND = dict(rows=8, dtype=1, qh=8, q=0x1000, k=0x11000, v=0x21000, out=0x31000, qr=512, qhs=64, kr=256, khs=64, vr=256, vhs=64, outr=512, ouths=64,
              pos=0x41000, axis=8, row=1, bits=32, res=0, slots=0x42000)


def split(change, base):
    c = {**CACHE, **{k[2:]: v for k, v in change.items() if k.startswith("c_")}}
    return {**base, **{k: v for k, v in change.items() if not k.startswith("c_")}}, c


@pytest.mark.parametrize("change,code,why", [
    (dict(dtype=3), EINVAL, "type"), (dict(dtype=2), EINVAL, "16-bit cache"), (dict(c_dim=128), EINVAL, "head size"), (dict(c_k=0), EINVAL, "null"),
    (dict(c_ks=2.0), EINVAL, "scales of 1"), (dict(c_dtype=4, c_ks=0.0), EINVAL, "positive"), (dict(c_dtype=4, c_vs=float("nan")), EINVAL, "positive"),
    (dict(c_dtype=3), EINVAL, "bf16, fp16 or e4m3"), (dict(c_pages=2**28), EOVERFLOW, "slots"), (dict(c_heads=0), EINVAL, "at least 1"),
    (dict(slots=0), EINVAL, "null"), (dict(out=0), EINVAL, "null"), (dict(slots=0x42002), EALIGN, "misaligned"), (dict(out=0x1002), EINVAL, "overlaps"),
    (dict(out=0x21000), EINVAL, "overlaps"), (dict(c_kt=0), EINVAL, "one another"), (dict(outr=0), EINVAL, "one another"), (dict(qh=-1), EINVAL, "heads"),
])
def test_append(change, code, why):
    a, c = split(change, APPEND)
    plan = ops.RopePlan(64)
    refused(lib.amap_rope_append(plan._h, APPEND_ARGS.pack(*a.values()) + CACHE_ARGS.pack(*c.values()), None), code, why)


ATTEND = dict(n=4, qh=8, dtype=1, max_pages=8, q=0x1000, out=0x11000, lse=0x21000, qr=512, qhs=64, outr=512, ouths=64, lser=8, table=0x31000, stride=8,
              lens=0x32000, scale=0.125, softcap=0.0, window=0, res=0, ws=0x400000, bytes=2**40, maps=0)


@pytest.mark.parametrize("change,code,why", [
    (dict(n=0), EINVAL, "requests"), (dict(qh=6), EINVAL, "multiple"), (dict(dtype=3), EINVAL, "type"), (dict(dtype=2), EINVAL, "16-bit cache"),
    (dict(c_dim=60), EUNSUPPORTED, "head size"), (dict(c_dim=264), EUNSUPPORTED, "head size"), (dict(c_dtype=4, c_dim=72), EUNSUPPORTED, "head size"),
    (dict(q=0), EINVAL, "null"), (dict(ws=0), EINVAL, "null"), (dict(max_pages=0), EINVAL, "rows"), (dict(stride=7), EINVAL, "rows"),
    (dict(max_pages=2**27, stride=2**27), EOVERFLOW, "2^31"), (dict(scale=float("nan")), EINVAL, "finite"), (dict(softcap=-1.0), EINVAL, "negative"),
    (dict(window=-1), EINVAL, "negative"), (dict(bytes=0), EINVAL, "workspace"), (dict(c_kt=260), EALIGN, "strides"), (dict(c_k=0x100008), EALIGN, "16 bytes"),
    (dict(lens=0x32002), EALIGN, "misaligned"), (dict(ws=0x400010), EALIGN, "misaligned"), (dict(out=0x1400), EINVAL, "overlap"),
])
def test_attend(change, code, why):
    a, c = split(change, ATTEND)
    refused(lib.amap_attend(ATTEND_ARGS.pack(*a.values()) + CACHE_ARGS.pack(*c.values()), None), code, why)


def test_cache_encode():
    out = ctypes.create_string_buffer(MAPS_ARGS.size)
    for change, code, why in ((dict(c_v=0), EINVAL, "null"), (dict(c_dim=260), EUNSUPPORTED, "head size"), (dict(c_kh=65), EALIGN, "strides"), (dict(c_v=0x200002), EALIGN, "16 bytes")):
        refused(lib.amap_cache_encode(CACHE_ARGS.pack(*split(change, {})[1].values()), out), code, why)
    refused(lib.amap_cache_encode(CACHE_ARGS.pack(*CACHE.values()), None), EINVAL, "null")
    # pages of 3 tokens have no maps; that is no refusal
    assert lib.amap_cache_encode(CACHE_ARGS.pack(*split(dict(c_page=3), {})[1].values()), out) == OK
    assert MAPS_ARGS.unpack(out.raw)[-1] == 0


def test_python_checks_its_tensors():
    """Tensors that are on no GPU, no tensors at all, and wrong numbers of them."""
    x = torch.zeros(4, 8, 64)
    i = torch.zeros(4, dtype=torch.int32)
    table = torch.zeros(4, 8, dtype=torch.int32)
    plan = ops.RopePlan(64)
    for call in (lambda: ops.PagedCache(torch.zeros(2, 16, 4, 64), torch.zeros(2, 16, 4, 64)),
                 lambda: ops.pages_extend(i, i, table, i, i[:1], 16, 4),
                 lambda: ops.pages_extend(i, i, None, i, i[:1], 16, 4),
                 lambda: ops.pages_release(torch.zeros(4, dtype=torch.bool), i, table, i, i[:1], 16),
                 lambda: plan.rotate([], i), lambda: plan.rotate([x], i), lambda: plan.rotate([x] * 5, i), lambda: plan.rotate(x, i),
                 lambda: plan.rotate([None], i), lambda: plan.rotate([x], i, outs=[])):
        with pytest.raises((ValueError, AttributeError)):
            call()
