"""The order of a chunk unit's work on its LDS stages (csrc/chunk_steps.h), run on the host: no stage is written in the
same stretch between two barriers in which it is read or written for another tile, as wavefronts may lie anywhere in it,
and what is read is the tile that was brought there in an earlier stretch."""
import ctypes
import os
import shutil
import subprocess

import pytest

from paper_2606_07577_amd import build

SOURCE = r"""
#include <cstdio>
#include <cstring>
#include <map>
#include <tuple>
#include <vector>
#include "chunk_steps.h"
namespace {
struct Access { int stretch; bool write; int tile; };
}
// Units of `tiles` key tiles from k0 on, of which those before mid are a memory's: the first fault's text, or "".
extern "C" const char* check(int k0, int tiles, int mid) {
  static char text[200];
  text[0] = 0;
  const auto fault = [&](const char* what, char buffer, int stage, int a, int b, int stretch) {
    if (!text[0]) std::snprintf(text, sizeof text, "%s: %c stage %d, tiles %d and %d, stretch %d", what, buffer, stage, a, b, stretch);
  };
  std::map<std::pair<char, int>, std::vector<Access>> log;
  int stretch = 0, at = k0, scores = -1, place = 0;
  const auto touch = [&](char buffer, int stage, bool write, int tile) {
    if (stage < 0 || stage > 3 || tile < k0 || tile >= k0 + tiles) return fault("out of range", buffer, stage, tile, tile, stretch);
    auto& all = log[{buffer, stage}];
    int held = -1;
    for (const Access& x : all) {
      if (x.stretch == stretch && (write || x.write) && !(write && x.write && x.tile == tile))
        fault("unordered", buffer, stage, x.tile, tile, stretch);
      if (x.write && x.stretch < stretch) held = x.tile;
    }
    if (!write && held != tile) fault("another tile", buffer, stage, held, tile, stretch);
    all.push_back({stretch, write, tile});
  };
  // a tail tile is copied from its fetch to the next barrier's wait, a memory tile goes to LDS in its store
  const auto fetch_k = [&](int t, int st) { if (t >= mid) touch('K', st, true, t); };
  const auto fetch_v = [&](int t, int st) { if (t >= mid) touch('V', st, true, t); };
  const auto store_k = [&](int t, int st) { if (t < mid) touch('K', st, true, t); };
  const auto store_v = [&](int t, int st) { if (t < mid) touch('V', st, true, t); };
  const auto first = [&](int st) { touch('K', st, false, k0); scores = k0; };
  const auto step = [&](auto memory, auto swapped, int t, int kst, int vst) {
    if (t != at || scores != t || decltype(swapped)::value != (place == 1)) fault("not in turn", 'S', place, t, scores, stretch);
    if (decltype(memory)::value != (t < mid)) fault("memory or tail", 'S', place, t, mid, stretch);
    touch('V', vst, false, t);
    if (t + 1 < k0 + tiles) touch('K', kst, false, t + 1);
    scores = ++at;
    place ^= 1;
  };
  const auto keep = [&]() { place = 0; };
  const auto barrier = [&]() { ++stretch; };
  const int k1 = k0 + tiles;
  omnimem::chunk_steps(k0, k1, mid < k0 ? k0 : mid > k1 ? k1 : mid, fetch_k, fetch_v, store_k, store_v, first, step, keep, barrier);
  if (at != k1) fault("steps left out", 'S', 0, at, k1, stretch);
  return text;
}
"""


@pytest.fixture(scope="module")
def check(tmp_path_factory):
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(hipcc):
        pytest.skip("hipcc not available")
    d = tmp_path_factory.mktemp("chunk_steps")
    (d / "check.hip").write_text(SOURCE)
    out = str(d / "check.so")
    flags = [f for f in build.FLAGS if f.startswith(("-std", "-f"))] + ["-O1", "-I", build.CSRC]
    res = subprocess.run([hipcc, "--cuda-host-only", *flags, "-shared", "-o", out, str(d / "check.hip")], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-2000:]
    lib = ctypes.CDLL(out)
    lib.check.restype = ctypes.c_char_p
    return lib.check


@pytest.mark.parametrize("k0", [0, 1, 5, 18])
@pytest.mark.parametrize("tiles", list(range(1, 14)) + [40, 41])
def test_stages_are_written_behind_a_barrier_after_their_last_use(check, k0, tiles):
    for mid in range(0, k0 + tiles + 3):           # all tail, both, all memory
        assert check(k0, tiles, mid) == b"", (k0, tiles, mid)
