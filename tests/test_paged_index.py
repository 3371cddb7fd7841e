"""Which rows of a cache in pages a query sees, which key tiles are taken and where their rows lie (csrc/paged.h), run on
the host against the definitions: every row that some query of a row tile sees is in one of its tiles, once; the rows of
a 16-row group are read from its page and inside it; no table is read past its last entry, and what no entry names is
read from page 0."""
import ctypes
import os
import random
import shutil
import subprocess

import numpy as np
import pytest

from oracle import operators_oracle as orc
from paper_2606_07577_amd import build

SOURCE = r"""
#include "paged.h"
using namespace omnimem;
template <int KT>
static int tiles(int nq, int nt, int window, int sinks, int i0, int i1, int tree, int* out, int* all) {
  const TailTiles x = tail_tiles_of<KT>(nq, nt, window, sinks, i0, i1, tree != 0);
  all[0] = x.all_from; all[1] = x.all_to;
  for (int t = 0; t < x.count && t < 4096; ++t) out[t] = tail_tile(x, t);
  return x.count;
}
extern "C" int tail_tiles(int kt, int nq, int nt, int window, int sinks, int i0, int i1, int tree, int* out, int* all) {
  return kt == 32 ? tiles<32>(nq, nt, window, sinks, i0, i1, tree, out, all) : kt == 64 ? tiles<64>(nq, nt, window, sinks, i0, i1, tree, out, all)
         : tiles<128>(nq, nt, window, sinks, i0, i1, tree, out, all);
}
extern "C" uint64_t seen64(int nq, int nt, int window, int sinks, int i, int tree, uint64_t mask, int key0) {
  return visible<uint64_t>(sight_of(nq, nt, window, i, tree != 0, mask), nt - nq, sinks, key0);
}
extern "C" uint32_t seen32(int nq, int nt, int window, int sinks, int i, int tree, uint64_t mask, int key0) {
  return visible<uint32_t>(sight_of(nq, nt, window, i, tree != 0, mask), nt - nq, sinks, key0);
}
// Byte of the 16 rows from key and their last one; the index of their entry; whether they have a page.
extern "C" int64_t place(int64_t page, uint32_t row, uint32_t n_pages, int shift, int nt, int32_t entry, int key, int32_t spare, int* last, int* index, int* there) {
  PagePool pool = {nullptr, nullptr, page, 0, row, n_pages, shift};
  const Place x = place_of(pool, nt, (uint32_t)entry, key, (uint32_t)spare);
  *last = x.last; *index = group_of(nt, key) >> shift; *there = x.there;
  return x.at;
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(hipcc):
        pytest.skip("hipcc not available")
    d = tmp_path_factory.mktemp("paged")
    (d / "paged.hip").write_text(SOURCE)
    out = str(d / "paged.so")
    flags = [f for f in build.FLAGS if f.startswith(("-std", "-f"))]
    res = subprocess.run([hipcc, "--cuda-host-only", *flags, "-O1", "-I", build.CSRC, "-I", os.path.join(build.ROOT, "include"), "-shared", "-o",
                          out, str(d / "paged.hip")], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-2000:]
    lib = ctypes.CDLL(out)
    lib.seen64.restype, lib.seen32.restype, lib.place.restype = ctypes.c_uint64, ctypes.c_uint32, ctypes.c_int64
    lib.seen64.argtypes = lib.seen32.argtypes = [ctypes.c_int] * 6 + [ctypes.c_uint64, ctypes.c_int]
    lib.place.argtypes = [ctypes.c_int64, ctypes.c_uint32, ctypes.c_uint32, ctypes.c_int, ctypes.c_int, ctypes.c_int32, ctypes.c_int, ctypes.c_int32] + [ctypes.c_void_p] * 3
    return lib


ALL = 1 << 30      # (the library's window 0)


def configs(count):
    rng = random.Random(11)
    for n in range(count):
        tree = n % 3 == 0
        nq = rng.randint(1, 64) if tree else rng.choice([1, 2, 7, 64, 150])
        nt = rng.randint(nq if tree else 1, 700)
        window, sinks = rng.choice([1, 5, 64, 100, 400, ALL]), rng.choice([0, 1, 4, 16, 33, 130, 900])
        masks = None
        if tree:
            masks = [rng.getrandbits(64) & rng.getrandbits(64) for _ in range(nq)]      # any bits: not a tree's only
            masks[0] = 0 if n % 2 else (1 << 64) - 1
        yield nq, nt, window, sinks, masks


def test_rows_that_are_seen(lib):
    for nq, nt, window, sinks, masks in configs(150):
        see = orc.paged_seen(nq, nt, 0 if window == ALL else window, sinks, masks)
        for i in range(nq):
            mask = masks[i] if masks else 0
            for key0 in range(0, (nt + 127) // 64 * 64 + 64, 32):
                want = sum(1 << j for j in range(64) if key0 + j < nt and see[i, key0 + j])
                tree = int(masks is not None)
                assert lib.seen64(nq, nt, window, sinks, i, tree, mask, key0) == want, (nq, nt, window, sinks, i, key0)
                assert lib.seen32(nq, nt, window, sinks, i, tree, mask, key0) == want & 0xFFFFFFFF


@pytest.mark.parametrize("kt", [32, 64, 128])
def test_tiles_hold_what_is_seen_once(lib, kt):
    out, both = np.zeros(4096, np.int32), np.zeros(2, np.int32)
    for nq, nt, window, sinks, masks in configs(200):
        see = orc.paged_seen(nq, nt, 0 if window == ALL else window, sinks, masks)
        rng = random.Random(nt)
        for _ in range(4):
            i0 = rng.randrange(nq)
            i1 = rng.randrange(i0, nq)
            n = lib.tail_tiles(kt, nq, nt, window, sinks, i0, i1, int(masks is not None), out.ctypes.data_as(ctypes.c_void_p),
                               both.ctypes.data_as(ctypes.c_void_p))
            tiles = out[:n].tolist()
            assert 0 <= n <= -(-nt // kt) and tiles == sorted(set(tiles)) and all(0 <= t and t * kt < nt for t in tiles)
            rows = np.flatnonzero(see[i0: i1 + 1].any(0))
            assert {r // kt for r in rows.tolist()} <= set(tiles)
            if both[0] < both[1]:                             # rows that every query sees
                assert see[i0: i1 + 1, both[0]: both[1]].all() and both[1] <= nt
            if window < nt and masks is None and i0 == i1:    # tiles without a row that is seen are few: one at each border
                used = {r // kt for r in rows.tolist()}
                assert len(set(tiles) - used) <= 1


def test_the_longest_tails_do_not_overflow(lib):
    out, both = np.zeros(4096, np.int32), np.zeros(2, np.int32)
    at = lambda *a: lib.tail_tiles(*a, out.ctypes.data_as(ctypes.c_void_p), both.ctypes.data_as(ctypes.c_void_p))
    assert at(128, 1, ALL, ALL, ALL, 0, 0, 0) == ALL // 128
    assert at(128, 1, ALL, 100, 4, 0, 0, 0) == 2 and out[:2].tolist() == [0, ALL // 128 - 1] and both.tolist() == [ALL - 100, ALL]
    assert at(64, ALL, 1, ALL, ALL, 0, 0, 0) == 0             # queries before the first tail row see nothing
    assert at(64, ALL, 1, ALL, ALL, 0, ALL - 1, 0) == 1
    assert lib.seen64(ALL, 1, ALL, ALL, 0, 0, 0, 0) == 0 and lib.seen64(ALL, 1, ALL, ALL, ALL - 1, 0, 0, 0) == 1
    assert lib.seen64(1, ALL, 3, 0, 0, 0, 0, ALL - 64) == 7 << 61


@pytest.mark.parametrize("page_rows", [16, 32, 64, 128, 256])
def test_places(lib, page_rows):
    last, index, there = (ctypes.c_int() for _ in range(3))
    shift, row, pages = page_rows.bit_length() - 1, 272, 9
    page = page_rows * row * 3
    for nt in (1, 15, 16, 17, 100, 256, 257, 1000):
        entries = -(-nt // page_rows)
        for key in range(0, nt + 256, 16):
            for entry in (0, 3, pages - 1, pages, -1, -2 ** 31, 2 ** 31 - 1):
                for spare in (-1, 5, pages, 0):
                    at = lib.place(page, row, pages, shift, nt, entry, key, spare, *(ctypes.byref(x) for x in (last, index, there)))
                    first, end = min(key, (nt - 1) // 16 * 16), (nt - 1) // 16 * 16
                    assert 0 <= index.value < entries and index.value == first // page_rows
                    assert there.value == (0 <= entry < pages)
                    if not there.value and 0 <= spare < pages:           # read as the rows with the last one
                        assert at == spare * page + end % page_rows * row and last.value == nt - 1 - end
                        continue
                    assert at == (entry if there.value else 0) * page + first % page_rows * row
                    assert last.value == min(15, nt - 1 - first) and first % page_rows + last.value < page_rows
    assert lib.place(1 << 40, (1 << 24) - 16, 2 ** 31 - 1, 8, 1 << 30, 50, 240, -1, *(ctypes.byref(x) for x in (last, index, there))) == \
        (50 << 40) + 240 * ((1 << 24) - 16)
