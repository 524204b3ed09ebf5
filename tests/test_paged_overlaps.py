"""Calls on a cache in pages whose outputs lie in what they read, or in one another, are refused; tensors between one another's rows are not (those calls get
as far as the launch, which fails without a GPU).  Nothing is read: addresses are numbers."""
import ctypes
import os

import pytest
import torch

from paper_2311_00368_b200 import build as b2sp_build

INVALID, CUDA = 1, 4
pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="calls that are taken would be launched")
FAR = 1 << 40


@pytest.fixture(scope="module")
def b():
    b2sp_build.build()
    from paper_2311_00368_b200 import binding
    return binding


def _pages(b, data, ld=64, sh=1024, sp=2048, pages=32, page=16):
    return b._PAGES(data, ld, sh, sp, pages, page)


def _tab(b, entries=FAR, ld=16, requests=3, width=16):
    return b._PAGE_TABLES(entries, ld, requests, width)


@pytest.mark.parametrize("bf16", [False, True])
def test_attention(b, bf16):
    M, H, Hkv, d, keep, e = 3, 4, 2, 64, 5, 2 if bf16 else 4
    fn = b.lib.b2sp_attention_paged_bf16 if bf16 else b.lib.b2sp_attention_paged
    q0, o0, lse0, seen, rows, tab, lists, k0, v0 = (FAR + (i << 30) for i in range(9))

    def f(q=q0, ldq=256, shq=64, o=o0, ldo=256, sho=64, lse=lse0, lists=lists, k=k0, v=v0, M=M, tab_ld=16):
        return fn(M, H, Hkv, d, q, ldq, shq, _pages(b, k), _pages(b, v), _tab(b, tab, tab_ld), rows, seen, lists, keep if lists else 0, 0.1, o, ldo, sho, lse,
                  1 << 20, 1 << 40, None)
    assert f() == f(lists=None) == CUDA
    for at, n in ((seen, 4 * M), (rows, 4 * M), (tab, 4 * 48), (lists, 4 * M * Hkv * keep)):
        for first, last in ((at, at + n - e), (at - e * (2 * 256 + 3 * 64 + 63), None)):         # O's first element in it, its last one
            assert f(o=first) == INVALID and (last is None or f(o=last) == INVALID)
        assert f(lse=at) == f(lse=at + n - 4) == f(lse=at - 4 * (M * H - 1)) == INVALID
        assert f(lse=at + n) == f(lse=at - 4 * M * H) == f(o=at + n) == CUDA
    assert f(lse=o0) == f(lse=o0 + e * 256) == f(lse=q0 + e * 512) == INVALID
    assert f(o=k0 + e * 2048 * 31) == f(o=v0 + e * 64) == f(lse=v0 + e * 2048) == INVALID
    # in the queries: themselves, with their strides; else nothing but what lies between their rows
    assert f(o=q0) == f(o=q0, ldq=768, ldo=768) == CUDA
    assert f(o=q0 + e) == f(o=q0 - e * 64) == f(o=q0 + e * 256) == f(o=q0, ldq=768) == f(o=q0, shq=0) == INVALID
    assert f(q=q0, ldq=768, o=q0 + e * 256, ldo=768) == f(q=q0, ldq=768, o=q0 + e * 512, ldo=768) == CUDA          # a projection's parts
    assert f(q=q0, ldq=512, shq=128, o=q0 + e * 64, ldo=512, sho=128) == CUDA                                      # every other head
    assert f(q=q0, ldq=512, shq=128, o=q0 + e * 65, ldo=512, sho=128) == f(q=q0, ldq=512, shq=128, o=q0 + e * 64, ldo=512) == INVALID
    assert f(M=1, o=q0, ldo=512) == CUDA and f(M=1, o=q0 + e * 256) == CUDA and f(M=1, o=q0 + e * 255) == INVALID
    # behind the entries of a table's rows
    assert f(lse=tab + 64, tab_ld=64) == CUDA and f(lse=tab + 256 - 44, tab_ld=64) == INVALID


@pytest.mark.parametrize("bf16", [False, True])
def test_write(b, bf16):
    fn, e = (b.lib.b2sp_paged_write_bf16, 2) if bf16 else (b.lib.b2sp_paged_write, 4)
    k0, v0, m0, ptr, lengths, tab = (FAR + (i << 30) for i in range(6))

    def f(k=_pages(b, k0), v=_pages(b, v0), means=_pages(b, m0, 0, 64, 128), ptr=ptr, lengths=lengths, tab=tab):
        return fn(4, 2, 64, 4096, 128, 64, 4096, 128, 64, ptr, lengths, _tab(b, tab), k, v, means, None)
    assert f() == f(means=None) == CUDA
    assert f(v=_pages(b, k0)) == f(v=_pages(b, k0 + e * 2048)) == f(v=_pages(b, k0 + e * 64)) == f(v=_pages(b, k0 - e * 2048 * 31)) == INVALID
    assert f(v=_pages(b, k0 + e * 2048 * 32)) == f(v=_pages(b, k0 - e * 2048 * 32)) == CUDA
    for at in (k0, k0 + e * 64, k0 + e * (2048 * 31 + 2040), v0, v0 - e * 128 * 31):
        assert f(means=_pages(b, at, 0, 64, 128)) == INVALID, at
    assert f(ptr=k0) == f(ptr=v0 + e * 2048 * 32 - 4) == f(ptr=m0 - 12) == f(lengths=k0 + e * 100) == f(tab=v0 - 4 * 47) == f(tab=m0) == INVALID
    # keys and values side by side: in a row, in a page, one row's heads after the other's; the mean behind a page's rows
    side = [dict(ld=128, sh=2048, sp=4096), dict(ld=64, sh=1024, sp=4096), dict(ld=256, sh=64, sp=4096), dict(ld=256, sh=128, sp=4096)]
    for layout, ahead in zip(side, (64, 2048, 128, 64)):
        assert f(k=_pages(b, k0, **layout), v=_pages(b, k0 + e * ahead, **layout)) == CUDA, layout
        assert f(k=_pages(b, k0, **layout), v=_pages(b, k0 + e * (ahead - 16 // e), **layout)) == INVALID, layout
    room = dict(ld=64, sh=17 * 64, sp=2 * 17 * 64)
    assert f(k=_pages(b, k0, **room), means=_pages(b, k0 + e * 16 * 64, 0, 17 * 64, 2 * 17 * 64)) == CUDA
    assert f(k=_pages(b, k0, **room), means=_pages(b, k0 + e * 15 * 64, 0, 17 * 64, 2 * 17 * 64)) == INVALID


def test_select(b):
    q0, m0, seen, tab, out = (FAR + (i << 30) for i in range(5))

    def f(out=out, m=_pages(b, m0, 0, 64, 128)):
        return b.lib.b2sp_paged_select(3, 4, 2, 64, q0, 256, 64, m, _tab(b, tab), None, seen, 4, 1, 1, out, 1 << 20, 1 << 30, None)
    assert f() == CUDA
    assert f(q0) == f(q0 + 4 * 767) == f(m0) == f(m0 + 4 * (32 * 128 - 1)) == f(m0 - 4 * 23) == f(seen) == f(tab) == INVALID
    assert f(q0 + 4 * 768) == f(m0 + 4 * 32 * 128) == CUDA


def test_tables_and_lists(b):
    names = ("lengths", "added", "free", "count", "out", "ptr", "rows", "seen", "slots", "counts", "tab")
    at = {n: FAR + (i << 20) for i, n in enumerate(names)}
    size = dict(lengths=12, added=12, free=128, count=4, out=12, ptr=16, rows=32, seen=32, slots=32, counts=16, tab=192)

    def tables(**other):
        a = {**at, **other}
        return b.lib.b2sp_paged_tables(_tab(b, a["tab"]), 32, 16, a["lengths"], a["added"], a["free"], 32, a["count"], 8, a["out"], a["ptr"], a["rows"], a["seen"],
                                       a["slots"], a["counts"], None)
    assert tables() == CUDA
    read = ("lengths", "added", "count")
    for x in names:
        for y in names:
            if x != y and not (x in read and y in read):
                assert tables(**{x: at[y]}) == tables(**{x: at[y] + size[y] - 4}) == INVALID, (x, y)
                assert tables(**{x: at[y] + size[y]}) == CUDA, (x, y)

    def lists(ptr=FAR, col=FAR + 4096):
        return b.lib.b2sp_paged_lists(3, _tab(b, FAR + (1 << 30)), 32, 16, None, FAR + (1 << 31), 9, ptr, col, None)
    assert lists() == CUDA
    assert lists(col=FAR) == lists(col=FAR + 12) == lists(ptr=FAR + 4096 + 32) == INVALID
    assert lists(col=FAR + 16) == CUDA


def test_tensors_between_one_another_s_rows():
    """The rule itself, against all bytes of small tensors."""
    import subprocess
    import tempfile
    csrc = os.path.join(os.path.dirname(b2sp_build.__file__), "csrc")
    with tempfile.TemporaryDirectory() as room:
        src, lib = os.path.join(room, "o.cpp"), os.path.join(room, "o.so")
        with open(src, "w") as f:
            f.write('#include "overlap.h"\nusing namespace b2sp;\nextern "C" int both(const long long *a, const long long *b)\n'
                    '{\n    const Spread x((const void *)a[0], a[1], {{a[2], a[3]}, {a[4], a[5]}, {a[6], a[7]}}), '
                    'y((const void *)b[0], b[1], {{b[2], b[3]}, {b[4], b[5]}, {b[6], b[7]}});\n    return share(x, y) + 2 * share(y, x) + 4 * (x == y);\n}\n')
        subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-I", csrc, "-o", lib, src], check=True)
        both = ctypes.CDLL(lib).both
    numbers = ctypes.c_longlong * 8
    import random
    rng = random.Random(1)

    def held(t):
        return {t[0] + i * t[3] + j * t[5] + k * t[7] + e for i in range(t[2]) for j in range(t[4]) for k in range(t[6]) for e in range(t[1])}
    met = 0
    for n in range(6000):
        x = [rng.randint(1, 200), rng.randint(1, 6)] + [rng.choice((rng.randint(1, 5), rng.randint(0, 60)))if i % 2 else rng.randint(1, 4) for i in range(6)]
        y = [x[0] + rng.randint(-80, 80) + 100] + x[1:] if n % 2 else [rng.randint(1, 200), rng.randint(1, 6)] + [rng.randint(0, 40) if i % 2 else rng.randint(0, 4) for i in range(6)]
        x[0] += 100
        truth, got = bool(held(x) & held(y)), both(numbers(*x), numbers(*y))
        assert got & 3 in (0, 3) and (got & 1 or not truth), (x, y)
        met += truth
        wide = sorted((s, m) for m, s in ((x[2], x[3]), (x[4], x[5]), (x[6], x[7])) if m > 1 and s)
        extent, nested = x[1], True
        for s, m in wide:
            nested &= s >= extent
            extent += (m - 1) * s
        if n % 2 and nested:                                              # the same strides, rows that do not overlap: exact
            assert bool(got & 1) == truth, (x, y)
    assert 1000 < met < 5000
