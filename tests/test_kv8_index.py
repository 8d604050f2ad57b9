"""The index arithmetic of the 8-bit cache's kernels (csrc/ot_kv8_index.h), compiled
for the host: every token, page and tile of a batch is some workgroup's and no index
leaves its tensor, whatever the lengths and tables on the device hold."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

from paper_2406_18832_amd import build_lib

SOURCE = r"""
#include "ot_kv8_index.h"
using namespace ot;
extern "C" {
void rows(int a, int b, long T, int *out) { auto r = kv8_rows(a, b, T); out[0] = r.row0; out[1] = r.n; }
long page_slot(long row, long b) { return kv8_page_slot(row, b); }
long page_slots(long T, long B) { return kv8_page_slots(T, B); }
long tile_slot(long row, long b, int unit) { return kv8_tile_slot(row, b, unit); }
long tile_slots(long T, long B, int unit) { return kv8_tile_slots(T, B, unit); }
void touch(long start, long n, long j, long *out) {
  auto t = kv8_touch(start, n, j); out[0] = t.col; out[1] = t.lo; out[2] = t.hi; }
long page(const int *table, long b, long col, long most, long pages) {
  return kv8_page(table, b, col, most, pages); }
void span(long len, long n, long i0, long rows, int causal, long window, int *out) {
  auto s = kv8_span(len, n, i0, rows, causal, window); out[0] = s.p0; out[1] = s.p1; }
long length(long len, long most) { return kv8_len(len, most); }
}
"""
L = ctypes.c_long


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("kv8")
    (d / "index.cpp").write_text(SOURCE)
    out = str(d / "index.so")
    run = subprocess.run([os.environ.get("CXX") or "g++", "-O1", "-std=c++17", "-Wall", "-Werror",
                          "-fsanitize=undefined", "-fno-sanitize-recover=undefined", "-static-libubsan",
                          "-shared", "-fPIC", "-I", build_lib.CSRC, str(d / "index.cpp"), "-o", out],
                         capture_output=True, text=True)
    if run.returncode:  # no static sanitizer runtime here
        run = subprocess.run([os.environ.get("CXX") or "g++", "-O1", "-std=c++17", "-Wall", "-Werror",
                              "-shared", "-fPIC", "-I", build_lib.CSRC, str(d / "index.cpp"),
                              "-o", out], capture_output=True, text=True)
    assert run.returncode == 0, run.stderr
    lib = ctypes.CDLL(out)
    for f in ("page_slot", "page_slots", "tile_slot", "tile_slots", "page", "length"):
        getattr(lib, f).restype = L
    return lib


def touch(lib, start, n, j):
    out = (L * 3)()
    lib.touch(L(start), L(n), L(j), out)
    return tuple(out)


def rows(lib, a, b, T):
    out = (ctypes.c_int * 2)()
    lib.rows(a, b, L(T), out)
    return out[0], out[1]


def span(lib, *args):
    out = (ctypes.c_int * 2)()
    lib.span(*[L(x) if i != 4 else ctypes.c_int(x) for i, x in enumerate(args)], out)
    return out[0], out[1]


def _batches():
    r = np.random.default_rng(5)
    for _ in range(150):
        B = int(r.integers(1, 70))
        n = np.where(r.random(B) < 0.3, r.integers(0, 2, B), r.integers(0, 300, B))
        start = np.where(r.random(B) < 0.3, 64 * r.integers(0, 4, B) - r.integers(0, 2, B),
                         r.integers(-100, 300, B))
        yield n, start
    yield np.array([64] * 5), np.array([63, 1, 0, 64, 62])
    yield np.array([2, 65, 66, 128, 1]), np.array([63, 63, 63, 1, -1])


def test_every_touched_page_has_a_slot_of_its_own(lib):
    for n, start in _batches():
        B, cu = len(n), np.concatenate(([0], np.cumsum(n)))
        T = int(cu[-1])
        first = [lib.page_slot(L(int(cu[b])), L(b)) for b in range(B)]
        total = lib.page_slots(L(T), L(B))
        seen = set()
        for s in range(total):
            b = sum(f <= s for f in first) - 1
            col, lo, hi = touch(lib, int(start[b]), int(n[b]), s - first[b])
            assert 0 <= lo < 64 and hi <= 64
            for t in range(lo, hi):
                assert (b, col * 64 + t) not in seen
                seen.add((b, col * 64 + t))
        assert seen == {(b, int(start[b]) + i) for b in range(B) for i in range(n[b])}


@pytest.mark.parametrize("unit,G", [(128, 1), (128, 5), (64, 3), (256, 1)])
def test_every_row_tile_has_a_slot_of_its_own(lib, unit, G):
    for n, _ in _batches():
        B, cu = len(n), np.concatenate(([0], np.cumsum(n)))
        first = [lib.tile_slot(L(int(cu[b]) * G), L(b), unit) for b in range(B)]
        total = lib.tile_slots(L(int(cu[-1]) * G), L(B), unit)
        seen = set()
        for s in range(total):
            b = sum(f <= s for f in first) - 1
            tiles = -(-int(n[b]) * G // unit)
            tile = tiles - 1 - (s - first[b])
            if 0 <= tile < tiles:
                assert (b, tile) not in seen
                seen.add((b, tile))
        assert seen == {(b, t) for b in range(B) for t in range(-(-int(n[b]) * G // unit))}


def test_rows_stay_in_the_batch(lib):
    for a, b, T, want in [(0, 5, 9, (0, 5)), (5, 5, 9, (5, 0)), (7, 3, 9, (7, 0)),
                          (-4, 3, 9, (0, 3)), (4, 1 << 30, 9, (4, 5)),
                          (-(1 << 31), (1 << 31) - 1, 9, (0, 9)), (20, 30, 9, (9, 0))]:
        assert rows(lib, a, b, T) == want


def test_pages_that_the_pool_does_not_have(lib):
    table = (ctypes.c_int * 6)(0, 7, -1, 8, 1 << 30, -(1 << 31))
    get = lambda b, col: lib.page(table, L(b), L(col), L(3), L(8))
    assert [get(0, c) for c in range(3)] == [0, 7, -1]
    assert [get(1, c) for c in range(3)] == [-1, -1, -1]
    assert get(0, 3) == -1 and get(0, -1) == -1 and get(1, 1 << 40) == -1


def test_lengths_stay_in_the_table(lib):
    assert [lib.length(L(n), L(3)) for n in (-5, 0, 191, 192, 193, (1 << 31) - 1)] == [0, 0, 191, 192,
                                                                                       192, 192]


def test_spans_hold_every_key_that_a_row_sees_and_no_page_without(lib):
    r = np.random.default_rng(6)
    for _ in range(600):
        length, n = int(r.integers(0, 400)), int(r.integers(1, 150))
        causal = int(r.random() < 0.7)
        window = int(r.integers(1, 200)) if causal and r.random() < 0.5 else 0
        i0 = int(r.integers(0, n))
        count = int(r.integers(1, n - i0 + 1))
        pos = length - n + np.arange(i0, i0 + count)[:, None]
        j = np.arange(length)[None, :]
        see = np.ones((count, length), bool)
        if causal:
            see &= j <= pos
        if window:
            see &= j > pos - window
        pages = np.flatnonzero(see.any(0)) // 64
        got = span(lib, length, n, i0, count, causal, window)
        want = (pages.min(), pages.max() + 1) if pages.size else (0, 0)
        if pages.size == 0:
            assert got[0] >= got[1]
        else:
            assert got == want, (length, n, causal, window, i0, count)


def _found(lib, cu, slot):
    """The sequence whose slot this is, as a wave counts them (64 at a time), or -1."""
    b = -1
    for b0 in range(0, len(cu) - 1, 64):
        n = sum(lib.page_slot(L(cu[x]), L(x)) <= slot for x in range(b0, min(b0 + 64, len(cu) - 1)))
        if n:
            b = b0 + n - 1
        if n < 64:
            break
    return b


def test_offsets_of_any_value_touch_rows_of_the_batch_only(lib):
    """Offsets that fall, or lie far outside the batch, can give a sequence slots far before
    its first one: no such slot has a place, and every place has a row of the sequence."""
    top, T = (1 << 31) - 1, 5
    r = np.random.default_rng(7)
    batches = [[-top - 1] * 100 + [top, -top - 1] + [top] * 29, [top] * 70 + [0],
               [0, top, -5, top, 3, 5], [-top - 1, 5], [7] * 130 + [top]]
    batches += [[int(x) for x in r.choice([-top - 1, -64, 0, 2, 5, 64, top], 140)] for _ in range(20)]
    far = 0
    for cu in batches:
        for slot in range(lib.page_slots(L(T), L(len(cu) - 1))):
            b = _found(lib, cu, slot)
            if b < 0:
                continue
            row0, n = rows(lib, cu[b], cu[b + 1], T)
            j = slot - lib.page_slot(L(cu[b]), L(b))
            far += j <= -(1 << 25)
            for start in (-top - 1, -1, 0, 64, 1 << 30, top - 63, top):
                col, lo, hi = touch(lib, start, n, j)
                assert 0 <= lo <= 64 and hi <= 64, (b, slot, start)
                if lo < hi:
                    assert row0 <= row0 + col * 64 + lo - start, (b, slot, start)
                    assert row0 + col * 64 + hi - start <= row0 + n, (b, slot, start)
    assert far > 0
