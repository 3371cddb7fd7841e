// Which tail rows of a cache in pages a query sees, the key tiles that a row
// tile takes of them and where 16 of its rows lie, apart from the work on them,
// so that it can be run on the host too.
#pragma once

#include <algorithm>

#include "attn.h"

namespace omnimem {

// A query at row p of the tail sees the rows j <= p with j > p - window or
// j < sinks.  p is n_t - n_q + i; with masks the last n_q rows are drafts, of
// which a query sees those of its mask alone, and it stands as many rows behind
// the last one before them as it sees.
struct Sight {
  int seen, lo;                // rows before the drafts: those below `seen` that are past `lo` or first ones
  uint64_t drafts;
};
template <typename U>
__host__ __device__ inline U bits_below(int n) {
  constexpr int W = 8 * (int)sizeof(U);
  return n >= W ? ~(U)0 : ~(~(U)0 << (n < 0 ? 0 : n));
}
__host__ __device__ inline int at_least_0(int n) { return n < 0 ? 0 : n; }
__host__ __device__ inline Sight sight_of(int nq, int nt, int window, int i, bool tree, uint64_t mask) {
  const int cached = nt - nq;
  Sight x;
  x.drafts = tree ? mask & bits_below<uint64_t>(nq) : 0;
  const int p = tree ? cached + __builtin_popcountll(x.drafts) - 1 : cached + i;
  x.seen = tree ? cached : at_least_0(p + 1);
  x.lo = at_least_0(p - window + 1);
  return x;
}
// Bit j: row key0 + j is seen (first_draft: n_t - n_q with masks, n_t without).
template <typename U>
__host__ __device__ inline U visible(const Sight& x, int first_draft, int sinks, int key0) {
  U bits = bits_below<U>(x.seen - key0) & (~bits_below<U>(x.lo - key0) | bits_below<U>(sinks - key0));
  const int first = first_draft - key0;
  if (x.drafts && first > -64 && first < 64) bits |= (U)(first >= 0 ? x.drafts << first : x.drafts >> -first);
  return bits;
}

// The key tiles (KT rows) of queries i0 .. i1: those with first rows, then those
// from the lowest window on; `skip` tiles lie between them and are neither
// looked up nor read.
struct TailTiles {
  int sink_tiles, skip, count;
  int all_from, all_to;        // rows that every one of the queries sees
};
template <int KT>
__host__ __device__ inline TailTiles tail_tiles_of(int nq, int nt, int window, int sinks, int i0, int i1, bool tree) {
  const int cached = nt - nq;
  const int p0 = tree ? cached - 1 : cached + i0, p1 = tree ? nt - 1 : cached + i1;   // (a draft stands between these)
  const int end = (int)(((int64_t)at_least_0(p1 + 1) + KT - 1) / KT), sink = (int)(((int64_t)sinks + KT - 1) / KT);
  const int lo = at_least_0(p0 - window + 1) / KT, low = lo < end ? lo : end;
  TailTiles x;
  x.sink_tiles = sink < low ? sink : low;
  x.skip = low - x.sink_tiles;
  x.count = end - x.skip;
  x.all_from = at_least_0(p1 - window + 1);
  x.all_to = tree ? cached : at_least_0(p0 + 1);
  return x;
}
__host__ __device__ inline int tail_tile(const TailTiles& x, int tt) { return tt + (tt >= x.sink_tiles ? x.skip : 0); }

// The 16 rows from `key` (a multiple of 16; behind the last row: those with it):
// their table entry's index, and with its value where they begin, in bytes from
// a head's first row on page 0, and how many rows follow the first that are not
// behind the last.  Without a page they are read all the same, and not used: as
// the rows with the last one, whose entry is `spare`, or if that is no page either
// (or not known) as those of page 0.
struct Place {
  int64_t at;
  int last;
  bool there;
};
__host__ __device__ inline int group_of(int nt, int key) {
  const int top = (nt - 1) & ~15;
  return key < top ? key : top;
}
constexpr uint32_t kNoPage = UINT32_MAX;
__host__ __device__ inline Place place_of(const PagePool& pool, int nt, uint32_t entry, int key, uint32_t spare) {
  int group = group_of(nt, key);
  Place x;
  x.there = entry < pool.n_pages;
  if (!x.there) {
    entry = spare < pool.n_pages ? spare : 0;
    if (spare < pool.n_pages) group = group_of(nt, nt);
  }
  x.at = (int64_t)entry * pool.page + (group & ((1 << pool.shift) - 1)) * (int64_t)pool.row;
  x.last = nt - 1 - group < 15 ? nt - 1 - group : 15;
  return x;
}

}  // namespace omnimem
