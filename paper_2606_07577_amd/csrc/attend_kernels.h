// Attention over a 4-bit memory and the tail rows behind it, which lie one
// after the other (attend.hip) or in the pages of a cache (attend_pages.hip).
//
// Every kernel makes one pass over the keys with a running maximum and sum:
// scores are formed transposed, S^T = K Q^T, so that a lane holds one query's
// scores, its maximum and its sum, and the weights leave the score's registers
// as they enter the second product, O^T = V^T P^T: an MFMA's sum runs over its
// keys in any order, so K and V are read in the order that the accumulator
// registers have.
#pragma once

#include <cmath>
#include <type_traits>

#include "../../include/omnimem.h"
#include "attn.h"
#include "chunk_steps.h"
#include "paged.h"

namespace omnimem {
namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));
using frag = bf16x8;

__device__ inline float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ inline int64_t elems(uint32_t units, int esz) { return (int64_t)units * (16 / esz); }

// Tail rows that query i sees.
__device__ inline int tail_seen(const QuerySeq& s, int causal, int i) {
  return causal ? min(max(s.nt - s.nq + i + 1, 0), s.nt) : s.nt;
}
template <int KT>
__host__ __device__ inline int tiles_of(int rows) { return (int)(((int64_t)rows + KT - 1) / KT); }

constexpr int kFewWaves = 4;     // wavefronts to a workgroup of the few-row kernels

// Tail rows in pages (see paged.h): the table's entry for the 16 rows from
// `key`, by a scalar load, and their place.
__device__ inline uint32_t entry_of(const PagePool& pool, const QuerySeq& s, int key) {
  typedef const __attribute__((address_space(4))) uint32_t scalar_t;
  return ((scalar_t*)(uintptr_t)s.k)[uniform(group_of(s.nt, key)) >> pool.shift];
}
__device__ inline Place place_at(const PagePool& pool, const QuerySeq& s, uint32_t entry, int key, uint32_t spare) {
  return place_of(pool, s.nt, (uint32_t)uniform((int)entry), uniform(key), (uint32_t)uniform((int)spare));
}

// ---------------------------------------------------------------------------
// Work of a unit.  Within a sequence the KV heads go fastest and the last row
// tiles, which see the most, come first: a causal tail's long units begin
// before its short ones, and as workgroups go to the 8 XCDs in turn, an XCD
// reads one head or a few.  Against heads one after the other, 32 neighbours to
// an XCD: 2048 queries of 28 heads over 4096 packed rows 172 -> 167 us, 8 x 1600
// queries of 16 heads over 8192 at width 64 536 -> 528, fp32 4 x 2048 over 6000
// tail rows 1564 -> 1429; 4 x 2048 over 6000 in bf16 213 -> 229.
// ---------------------------------------------------------------------------
struct Unit {
  int s, g, rt;              // sequence, KV head, row tile
  int rows;                  // query rows of the head (G * n_q)
  int k0, k1;                // key tiles
  int mem_tiles;             // of the sequence
  int slot;                  // partial, or -1: the result is final
  int split, splits;         // its share of the row tile
  TailTiles tail;            // in pages
  bool holes;                // and some of them without a page
};
// Row tile's tail key tile tt of those that it takes.
template <class A>
__device__ inline int tail_tile(const Unit& x, int tt) {
  if constexpr (A::kPaged) return tail_tile(x.tail, tt);
  return tt;
}
// The last sequence whose entry of `first` is at most u (lane-parallel).
template <int N>
__device__ inline int seq_of(const int32_t (&first)[N], int n, int u) {
  if constexpr (N == 1) return 0;
  const int lane = threadIdx.x & 63;
  const int v = lane < n ? first[lane] : INT32_MAX;
  return uniform(__popcll(__ballot(v <= u)) - 1);
}
template <int R, int KT, int WAVES, class A>    // WAVES: that go through the key tiles in turn
__device__ inline Unit unit_of(const A& a, int u) {
  Unit x;
  int tile;
  x.split = 0;
  x.splits = 1;
  x.slot = -1;
  if (a.whole > 0) {
    tile = u;
    if (u >= a.whole) {
      x.splits = a.seq[0].splits;
      x.slot = u - a.whole;
      tile = a.whole + x.slot / x.splits;
      x.split = x.slot % x.splits;
    }
    x.s = seq_of(a.unit0, a.n_seqs, tile);
    tile -= a.unit0[x.s];
  } else {
    x.s = seq_of(a.unit0, a.n_seqs, u);
    u -= a.unit0[x.s];
    x.splits = a.seq[x.s].splits;
    if (x.splits > 1) x.slot = a.seq[x.s].slot0 + u;
    tile = u / x.splits;
    x.split = u % x.splits;
  }
  const QuerySeq& s = a.seq[x.s];
  x.g = tile % a.h_kv;
  x.rt = s.row_tiles - 1 - tile / a.h_kv;
  x.rows = a.group * s.nq;
  x.mem_tiles = tiles_of<KT>(s.nm);
  const int last = (min((x.rt + 1) * R, x.rows) - 1) / a.group;
  int tail_tiles;
  if constexpr (A::kPaged) {
    x.tail = tail_tiles_of<KT>(s.nq, s.nt, a.window, a.sinks, x.rt * R / a.group, last, s.v != nullptr);
    x.holes = false;
    tail_tiles = x.tail.count;
  } else {
    tail_tiles = tiles_of<KT>(tail_seen(s, a.causal, last));
  }
  const int tiles = x.mem_tiles + tail_tiles;
  if constexpr (WAVES == 1) {
    x.k0 = (int)((int64_t)tiles * x.split / x.splits);
    x.k1 = (int)((int64_t)tiles * (x.split + 1) / x.splits);
  } else {                   // as many for each wavefront
    const int64_t share = ((tiles + x.splits - 1) / x.splits + WAVES - 1) / WAVES * WAVES;
    x.k0 = (int)min((int64_t)tiles, share * x.split);
    x.k1 = (int)min((int64_t)tiles, share * (x.split + 1));
  }
  return x;
}

// One query row of a tile: where its query is, and the tail rows that it sees.
struct Row {
  bool live;
  int i, h, seen;
  Sight sight;               // in pages
};
template <class A>
__device__ inline Row row_of(const A& a, const QuerySeq& s, const Unit& x, int row) {
  Row r;
  r.live = row < x.rows;
  r.i = r.live ? row / a.group : 0;
  r.h = x.g * a.group + (r.live ? row - r.i * a.group : 0);
  if constexpr (A::kPaged) {
    const uint64_t mask = s.v && r.live ? gload<uint64_t>(static_cast<const uint64_t*>(s.v) + r.i) : 0;
    r.sight = sight_of(s.nq, s.nt, a.window, r.i, s.v != nullptr, mask);
    if (!r.live) r.sight.seen = 0;
  } else {
    r.seen = r.live ? tail_seen(s, a.causal, r.i) : 0;
  }
  return r;
}
// Bit j: the query sees tail row key0 + j (in pages; whether it has a page is
// not looked at).
template <typename U, class A>
__device__ inline U visible(const A& a, const QuerySeq& s, const Row& row, int key0) {
  return visible<U>(row.sight, s.nt - s.nq, a.sinks, key0);
}
// Whether some 16 of the unit's tail rows have no page: look() asks for the
// entries of the first 256 sixteens (a lane to each), found() takes them, and
// those behind, once what was asked for later is here too (with a wait for them
// before the first rows 4096 queries over a window of 4096 take 272 us, not 270).
template <int KT, class A>
struct Holes {
  static constexpr int GROUPS = KT / 16, FIRST = 4;
  int t0, n;
  uint32_t entry[FIRST];
  __device__ inline uint32_t at(const A& a, const QuerySeq& s, const Unit& x, int i) const {
    const int key = tail_tile<A>(x, t0 + i / GROUPS) * KT + i % GROUPS * 16;
    return gload<uint32_t>(static_cast<const uint32_t*>(s.k) + (group_of(s.nt, key) >> a.pool.shift));
  }
  __device__ inline void look(const A& a, const QuerySeq& s, const Unit& x) {
    t0 = max(x.k0 - x.mem_tiles, 0);
    n = (x.k1 - x.mem_tiles - t0) * GROUPS;
#pragma unroll
    for (int j = 0; j < FIRST; ++j) entry[j] = n > 0 ? at(a, s, x, min(j * 64 + (int)(threadIdx.x & 63), n - 1)) : 0;
  }
  __device__ inline bool found(const A& a, const QuerySeq& s, const Unit& x) const {
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < FIRST; ++j) top = max(top, entry[j]);
    for (int i = FIRST * 64 + (int)(threadIdx.x & 63); i < n; i += 64) top = max(top, at(a, s, x, i));
    return __any(top >= a.pool.n_pages);
  }
};
// Bits of a tile's rows that have a page.
template <typename U, class A>
__device__ inline U paged_bits(const A& a, const QuerySeq& s, int key0) {
  U bits = 0;
#pragma unroll
  for (int i = 0; i < (int)sizeof(U) / 2; ++i)
    if (entry_of(a.pool, s, key0 + i * 16) < a.pool.n_pages) bits |= (U)0xFFFF << (16 * i);
  return bits;
}

__device__ inline void put4(uint16_t* p, floatx4 x) { *reinterpret_cast<uint2*>(p) = make_uint2(round2(x[0], x[1]), round2(x[2], x[3])); }
__device__ inline void put4(float* p, floatx4 x) { *reinterpret_cast<floatx4*>(p) = x; }
__device__ inline void put1(uint16_t* p, float x) { *p = (uint16_t)round2(x, 0.0f); }
__device__ inline void put1(float* p, float x) { *p = x; }
// Partials pass between workgroups of one launch: they are written to and read
// from the device's coherent memory (8 bytes at a time, past the XCD's L2), and
// a wait for the writes orders them before the count of the units that wrote
// theirs.  A release of all that the L2 holds, and an acquire, are not needed:
// with them at the end of each unit 32 users' tokens took 58 us instead of 50.
__device__ inline void share8(float* p, float x, float y) {
  const uint64_t v = (uint64_t)__float_as_uint(y) << 32 | __float_as_uint(x);
  __hip_atomic_store(reinterpret_cast<uint64_t*>(p), v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ inline floatx2 shared8(const float* p) {
  const uint64_t v = __hip_atomic_load(reinterpret_cast<const uint64_t*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return floatx2{__uint_as_float((uint32_t)v), __uint_as_float((uint32_t)(v >> 32))};
}
// The larger of a lane's value and that of the lane 32 (16) away.
__device__ inline float max32(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ inline float max16(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
// A row's sums over the sum of its weights; 0 if it has none, whatever the
// values are that weights of 0 were multiplied with.
__device__ inline floatx4 over(floatx4 y, float l) { return l == 0.0f ? floatx4{} : y * (1.0f / l); }
__device__ inline float log_of(float m, float l) { return l == 0.0f ? -INFINITY : (m + log2f(l)) * kLn2; }

// ---------------------------------------------------------------------------
// Rows that a query does not see have weight 0, but the matrix cores multiply
// it with what the row holds, and 0 times an infinity or NaN is NaN.  So do the
// rows behind the last one in its tile, which are copies of it.  A unit whose
// sums are not finite forms the rows again that have either among its keys, each
// by one wavefront over the keys that the row sees, and writes them over what
// it wrote.  A row whose weights are NaN has NaN everywhere by right, and one
// with finite values alone behind the keys that it sees has what it sees: they
// stay.  (1000 queries of 8 heads of width 128 over 2001 keys, 34 us: where all
// of them are NaN 34, where they are formed again for an infinity in the last
// value, one after the other in a wavefront, 4800.)
// ---------------------------------------------------------------------------
template <int KT, class A>
__device__ inline bool sees_all(const QuerySeq& s, const Unit& x, const Row& row) {     // whole tiles
  if constexpr (A::kPaged) {
    const int64_t begin = (int64_t)tail_tile<A>(x, max(x.k0 - x.mem_tiles, 0)) * KT;
    const int64_t end = (int64_t)tail_tile<A>(x, x.k1 - x.mem_tiles - 1) * KT + KT;
    return !s.v && !x.holes && row.sight.lo <= begin && row.sight.seen >= end;
  }
  return row.seen >= (int64_t)(x.k1 - x.mem_tiles) * KT;
}
template <int D, typename T>
__device__ inline void channels(const T* p, int lane, float (&y)[D / 64]) {
#pragma unroll
  for (int i = 0; i < D / 64; ++i) {
    if constexpr (sizeof(T) == 2) y[i] = __uint_as_float((uint32_t)gload<uint16_t>(p + lane + i * 64) << 16);
    else y[i] = gload<float>(p + lane + i * 64);
  }
}
template <typename T, int D, int R, int KT, class A>
__device__ __forceinline__ void form_again(const A& a, const QuerySeq& s, const Unit& x, int r, float m, float l) {
  using B = MemBlock<D>;
  constexpr int E = (int)sizeof(T), C = D / 64;
  const int lane = threadIdx.x & 63;
  const Row row = row_of(a, s, x, x.rt * R + r);
  if (!row.live || sees_all<KT, A>(s, x, row) || l != l) return;
  // (at most 2^30 rows and a tile; copies of the last row have its values)
  const int begin = max(x.k0 - x.mem_tiles, 0) * KT, end = min((x.k1 - x.mem_tiles) * KT, s.nt);
  const int64_t rs = elems(s.kv_rs, E);
  const T* vp = static_cast<const T*>(s.v) + x.g * elems(s.kv_hs, E);
  // (in pages) the unit's tail rows: f(K row, V row, it is seen)
  const auto each = [&](auto&& f) __attribute__((always_inline)) {
    if constexpr (A::kPaged) {
      const uint32_t spare = x.holes ? entry_of(a.pool, s, s.nt) : kNoPage;
      for (int tt = max(x.k0 - x.mem_tiles, 0); tt < x.k1 - x.mem_tiles; ++tt)
        for (int key0 = tail_tile<A>(x, tt) * KT, b = 0; b < KT; b += 16) {
          const Place at = place_at(a.pool, s, entry_of(a.pool, s, key0 + b), key0 + b, spare);
          const uint32_t seen = at.there ? visible<uint32_t>(a, s, row, key0 + b) : 0u;
          for (int j = 0; j < 16; ++j) {
            const int64_t byte = at.at + x.g * a.pool.head + min(j, at.last) * (int64_t)a.pool.row;
            f(reinterpret_cast<const T*>(a.pool.k + byte), reinterpret_cast<const T*>(a.pool.v + byte), (seen >> j & 1u) != 0);
          }
        }
    }
  };
  float zero = 0.0f;
  const auto odd = [&](const T* p) __attribute__((always_inline)) {
    float v[C];
    channels<D>(p, lane, v);
#pragma unroll
    for (int i = 0; i < C; ++i) zero = __builtin_fmaf(v[i], 0.0f, zero);
  };
  if constexpr (A::kPaged)
    each([&](const T*, const T* v, bool seen) __attribute__((always_inline)) { if (!seen) odd(v); });
  else
    for (int j = min(max(row.seen, begin), s.nt - 1); j < end; ++j) odd(vp + j * rs);
  if (!__any(zero != 0.0f)) return;
  const float ref = m == -INFINITY ? 0.0f : m;
  float q[C], o[C] = {};
  channels<D>(static_cast<const T*>(s.q) + row.h * elems(s.q_hs, E) + row.i * elems(s.q_rs, E), lane, q);
  const auto add = [&](const float (&k)[C], const float (&v)[C]) __attribute__((always_inline)) {
    float dot = 0.0f;
#pragma unroll
    for (int i = 0; i < C; ++i) dot += q[i] * k[i];
#pragma unroll
    for (int e = 1; e < 64; e *= 2) dot += __shfl_xor(dot, e);
    const float p = exp2_(dot * s.scale_log2 - ref);
#pragma unroll
    for (int i = 0; i < C; ++i) o[i] += p * v[i];
  };
  const int64_t mem_end = min((int64_t)s.nm, (int64_t)x.k1 * KT);
  for (int64_t j = (int64_t)x.k0 * KT; j < mem_end; ++j) {
    const char* blk = s.mem + x.g * ((int64_t)s.mem_hs * 16) + j / kMemRows * B::BYTES;
    const int t = (int)(j % kMemRows);
    float k[C], v[C], y[8];
#pragma unroll
    for (int i = 0; i < C; ++i) {
      const int c = lane + i * 64;
      values8(gload<uint8_t>(blk + t * (D / 2) + c / 2), gload<uint8_t>(blk + B::k_scale(t, c >> 5)), y);
      k[i] = c & 1 ? y[1] : y[0];
      values8(gload<uint8_t>(blk + B::V + c * 16 + t / 2), gload<uint8_t>(blk + B::v_scale(c)), y);
      v[i] = t & 1 ? y[1] : y[0];
    }
    add(k, v);
  }
  const T* kp = static_cast<const T*>(s.k) + x.g * elems(s.kv_hs, E);
  const auto tail_row = [&](const T* kr, const T* vr) __attribute__((always_inline)) {
    float k[C], v[C];
    channels<D>(kr, lane, k);
    channels<D>(vr, lane, v);
    add(k, v);
  };
  if constexpr (A::kPaged)
    each([&](const T* kr, const T* vr, bool seen) __attribute__((always_inline)) { if (seen) tail_row(kr, vr); });
  else
    for (int j = begin; j < min(row.seen, end); ++j) tail_row(kp + j * rs, vp + j * rs);
  const float inv = 1.0f / l;
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");   // (after what the workgroup wrote there)
#pragma unroll
  for (int i = 0; i < C; ++i) {
    const int c = lane + i * 64;
    if (x.slot >= 0) __hip_atomic_store(a.part_o + ((int64_t)x.slot * R + r) * D + c, o[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    else put1(static_cast<T*>(s.out) + row.h * elems(s.out_hs, E) + row.i * elems(s.out_rs, E) + c, l == 0.0f ? 0.0f : o[i] * inv);
  }
}
// The same for a wavefront's own 32 rows (a lane each, twice).
template <typename T, int D, int R, int KT, class A>
__device__ __forceinline__ void form_own(const A& a, const QuerySeq& s, const Unit& x, const Row& row, int r0,
                                const floatx16 (&o)[D / 32], float m, float l) {
  if (x.k1 <= x.mem_tiles) return;
  float zero = 0.0f;
#pragma unroll
  for (int c = 0; c < D / 32; ++c)
#pragma unroll
    for (int e = 0; e < 16; ++e) zero = __builtin_fmaf(o[c][e], 0.0f, zero);
  uint64_t odd = __ballot(zero != 0.0f && row.live && !sees_all<KT, A>(s, x, row));
  for (odd = (odd | odd >> 32) & 0xFFFFFFFFu; odd; odd &= odd - 1) {
    const int r = __builtin_ctzll(odd);
    form_again<T, D, R, KT>(a, s, x, r0 + r, __shfl(m, r), __shfl(l, r));
  }
}

// The end of a unit whose wavefronts have sums of their own, in LDS [WAVES]
// [R][ROW], taken by their share of the row's maximum: added up, they go to the
// output or, with more than one unit to the row tile, to a partial.  The last
// unit of a row tile to write its partial joins them all (`arrived` counts
// them, and is 0 again afterwards), in the order of the keys, unless that is
// more work than a kernel for it (see kJoinBatches).
struct Joint {
  float2 ml[64];             // (maximum, sum) of a row
  int flag[64];              // its sums are not finite
  int last;
};
template <typename T, int D, int R, int KT, int ROW, int WAVES, class A>
__device__ __forceinline__ void finish(const A& a, const QuerySeq& s, const Unit& x, float* ob, Joint* joint) {
  static_assert(R <= 64, "rows of a Joint");
  constexpr int E = (int)sizeof(T), THREADS = 64 * WAVES, TPR = D / 4;
  const int tid = threadIdx.x, live = min(R, x.rows - x.rt * R);
  const auto put_row = [&](int r, int c, floatx4 y, float l) __attribute__((always_inline)) {
    const Row row = row_of(a, s, x, x.rt * R + r);
    put4(static_cast<T*>(s.out) + row.h * elems(s.out_hs, E) + row.i * elems(s.out_rs, E) + c, over(y, l));
  };
  const auto put_lse = [&](int r, float m, float l) __attribute__((always_inline)) {
    const Row row = row_of(a, s, x, x.rt * R + r);
    if (s.lse) s.lse[row.h * (int64_t)s.lse_hs + row.i] = log_of(m, l);
  };
  bool odd = false;
  if (tid < R) joint->flag[tid] = 0;
  __syncthreads();
  for (int e = tid; e < live * TPR; e += THREADS) {
    const int r = e / TPR, c = e % TPR * 4;
    floatx4 y = floatx4{};
#pragma unroll
    for (int w = 0; w < WAVES; ++w) y += *reinterpret_cast<const floatx4*>(ob + (w * R + r) * ROW + c);
    if (x.slot >= 0) {
      float* p = a.part_o + ((int64_t)x.slot * R + r) * D + c;
      if (a.joined) {
        share8(p, y[0], y[1]);
        share8(p + 2, y[2], y[3]);
      } else {
        put4(p, y);
      }
    } else {
      put_row(r, c, y, joint->ml[r].y);
    }
    if (x.k1 > x.mem_tiles && (y[0] + y[1] + y[2] + y[3]) * 0.0f != 0.0f) {
      joint->flag[r] = 1;
      odd = true;
    }
  }
  if (tid < live) {
    const float2 ml = joint->ml[tid];
    if (x.slot >= 0) share8(&a.part_ml[(int64_t)x.slot * R + tid].x, ml.x, ml.y);
    else put_lse(tid, ml.x, ml.y);
  }
  bool again = true;                                       // (one look at all flags where no row has one)
  if constexpr (A::kPaged) again = __syncthreads_or(odd) != 0;
  else __syncthreads();
  for (int r = wave_id(); again && r < live; r += WAVES)
    if (uniform(joint->flag[r])) form_again<T, D, R, KT>(a, s, x, r, joint->ml[r].x, joint->ml[r].y);
  if (x.slot < 0 || !a.joined) return;

  const int first = x.slot - x.split;
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");         // (this wavefront's part of the partial is in coherent memory)
  __syncthreads();
  if (tid == 0)
    joint->last = __hip_atomic_fetch_add(a.arrived + first, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == x.splits - 1;
  __syncthreads();
  if (!joint->last) return;
  if (tid == 0) __hip_atomic_store(a.arrived + first, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  // `shares` threads to a row's 4 channels, with 8 partials on their way each
  const int items = live * TPR;
  int shares = 1;
  while (2 * shares * items <= THREADS && shares < x.splits) shares *= 2;
  floatx4* os = reinterpret_cast<floatx4*>(ob);            // [shares][items], and their statistics
  float2* mls = reinterpret_cast<float2*>(os + THREADS);
  for (int e = tid; e < items * shares; e += THREADS) {
    const int item = e % items, r = item / TPR, c = item % TPR * 4;
    const float* ml = &a.part_ml[(int64_t)first * R + r].x;
    const float* po = a.part_o + ((int64_t)first * R + r) * D + c;
    float m = -INFINITY, l = 0.0f;
    floatx4 o = floatx4{};
    for (int p0 = e / items; p0 < x.splits; p0 += 8 * shares) {
      floatx2 y[8], z[8][2];
#pragma unroll
      for (int b = 0; b < 8; ++b) {
        const int64_t p = min(p0 + b * shares, x.splits - 1);
        y[b] = shared8(ml + p * R * 2);
        z[b][0] = shared8(po + p * R * D);
        z[b][1] = shared8(po + p * R * D + 2);
      }
#pragma unroll
      for (int b = 0; b < 8; ++b) {
        if (p0 + b * shares >= x.splits) break;
        const float m2 = fmaxf(m, y[b][0]), ref = m2 == -INFINITY ? 0.0f : m2;
        const float was = exp2_(m - ref), is = exp2_(y[b][0] - ref);
        l = l * was + y[b][1] * is;
        o = o * was + floatx4{z[b][0][0], z[b][0][1], z[b][1][0], z[b][1][1]} * is;
        m = m2;
      }
    }
    if (shares == 1) {
      put_row(r, c, o, l);
      if (c == 0) put_lse(r, m, l);
    } else {
      os[e] = o;
      mls[e] = make_float2(m, l);
    }
  }
  if (shares == 1) return;
  __syncthreads();
  for (int e = tid; e < items; e += THREADS) {
    const int r = e / TPR, c = e % TPR * 4;
    float m = -INFINITY, l = 0.0f;
    for (int p = 0; p < shares; ++p) m = fmaxf(m, mls[e + p * items].x);
    const float ref = m == -INFINITY ? 0.0f : m;
    floatx4 o = floatx4{};
    for (int p = 0; p < shares; ++p) {
      const float w = exp2_(mls[e + p * items].x - ref);
      l += mls[e + p * items].y * w;
      o += os[e + p * items] * w;
    }
    put_row(r, c, o, l);
    if (c == 0) put_lse(r, m, l);
  }
}

// A wavefront's sums of 32 rows (lane: row `r` of the tile, channels by
// accumulator register) to their partial or, divided, to the output.
template <typename T, int D, int R, class A>
__device__ inline void write_rows(const A& a, const QuerySeq& s, const Unit& x, const Row& row, int r, int half,
                                  const floatx16 (&o)[D / 32], float m, float l) {
  constexpr int E = (int)sizeof(T);
  if (x.slot >= 0) {
    const int64_t at = (int64_t)x.slot * R + r;
    if (half == 0) a.part_ml[at] = make_float2(m, l);
#pragma unroll
    for (int c = 0; c < D / 32; ++c)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        put4(a.part_o + at * D + c * 32 + e * 8 + half * 4, floatx4{o[c][4 * e], o[c][4 * e + 1], o[c][4 * e + 2], o[c][4 * e + 3]});
  } else if (row.live) {
    T* out = static_cast<T*>(s.out) + row.h * elems(s.out_hs, E) + row.i * elems(s.out_rs, E);
    if (half == 0 && s.lse) s.lse[row.h * (int64_t)s.lse_hs + row.i] = log_of(m, l);
#pragma unroll
    for (int c = 0; c < D / 32; ++c)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        put4(out + c * 32 + e * 8 + half * 4, over(floatx4{o[c][4 * e], o[c][4 * e + 1], o[c][4 * e + 2], o[c][4 * e + 3]}, l));
  }
}

// ---------------------------------------------------------------------------
// fp32, few rows: 32 query rows to a unit, whose key tiles of 32 rows go round
// the four wavefronts, each with sums of its own that are joined at the end.  A
// tile goes from memory to registers and from there to the MFMAs: lane (i, h) =
// (lane % 32, lane / 32) reads channels 8 j + 4 h .. of K row i, and of V
// channel i of every 32 the rows that its weights are of, 8 e + 4 h .. of a
// memory block's codes (16 bytes have a channel's 32 rows).  The next tile's K
// is on its way during the weights and V's products, V during K's.  The MFMAs
// bound a long cache (32 rows at least, of which a token has a head's queries:
// 8 sequences of 7 rows and 4 heads of width 128 over 4096 tail rows, 134 MB,
// 38 us, 3.6 TB/s; over memory rows 36), latency a short one (7 rows over 4096
// memory rows 16 us).
// ---------------------------------------------------------------------------
template <int D>
struct F32 {
  static constexpr int R = 32, KT = 32, WAVES = 4;
  static constexpr int ROW = D + 4;                        // padded LDS row
  static constexpr int LDS = 4 * R * ROW * 4 + 4 * R * 8 + (int)sizeof(Joint);
};
// Four values of a word of codes: the low or (h) high half.
__device__ inline floatx4 values4(uint32_t w, int h, uint32_t byte) {
  const float s = scale_of(byte);
  const floatx2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w >> (16 * h), s, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w >> (16 * h), s, 1);
  return floatx4{a[0], a[1], b[0], b[1]};
}

template <int D, class A>
__global__ __launch_bounds__(256) void attend_f32(A a) {
  using P = F32<D>;
  using M = Mfma<float>;
  constexpr int R = P::R, KT = P::KT, ROW = P::ROW, NCT = D / 32;
  using B = MemBlock<D>;
  extern __shared__ __align__(16) char lds[];
  float* ob = reinterpret_cast<float*>(lds);               // [4][R][ROW]
  float2* ml = reinterpret_cast<float2*>(ob + 4 * R * ROW); // [4][R]
  Joint* joint = reinterpret_cast<Joint*>(ml + 4 * R);
  const Unit x = unit_of<R, KT, kFewWaves>(a, blockIdx.x);
  const QuerySeq& s = a.seq[x.s];
  const int lane = threadIdx.x & 63, wave = wave_id(), half = lane >> 5, col = lane & 31;
  const Row row = row_of(a, s, x, x.rt * R + col);
  const float* qp = static_cast<const float*>(s.q) + row.h * elems(s.q_hs, 4) + row.i * elems(s.q_rs, 4);
  floatx4 q[D / 8];
#pragma unroll
  for (int j = 0; j < D / 8; ++j) q[j] = row.live ? gload<floatx4>(qp + 8 * j + 4 * half) : floatx4{};
  uint32_t rsb = s.kv_rs * 16u;                            // row stride in bytes, below 2^24
  const char* kp = static_cast<const char*>(s.k) + x.g * ((int64_t)s.kv_hs * 16);
  const char* vp = static_cast<const char*>(s.v) + x.g * ((int64_t)s.kv_hs * 16);
  if constexpr (A::kPaged) {
    rsb = a.pool.row;
    kp = a.pool.k + x.g * a.pool.head;
    vp = a.pool.v + x.g * a.pool.head;
  }
  const char* data = s.mem + x.g * ((int64_t)s.mem_hs * 16);
  const int mem_tiles = x.mem_tiles, nt = s.nt, nm = s.nm;

  uint4 kr[D / 8];                                         // a tile's rows, or (the first) codes
  uint32_t vr[16 * NCT], kb[NCT], vb[NCT];
  uint32_t entry[2] = {};                                  // in pages: of the tile to be loaded
  Place place[2] = {};                                     // and of the one that is
  const auto look = [&](int t) __attribute__((always_inline)) {
    if constexpr (A::kPaged)
#pragma unroll
      for (int b = 0; b < 2; ++b) entry[b] = entry_of(a.pool, s, tail_tile<A>(x, t - mem_tiles) * KT + b * 16);
  };
  const auto load_k = [&](int t) __attribute__((always_inline)) {
    if (t < mem_tiles) {
      const char* block = data + (int64_t)t * B::BYTES;
#pragma unroll
      for (int j = 0; j < NCT; ++j) {
        kr[j] = gload16(block + (uint32_t)(col * (D / 2) + j * 16));
        kb[j] = gload<uint8_t>(block + (uint32_t)B::k_scale(col, j));
      }
    } else if constexpr (A::kPaged) {
      if (t - 4 < mem_tiles) look(t);                      // (behind a memory tile)
#pragma unroll
      for (int b = 0; b < 2; ++b) place[b] = place_at(a.pool, s, entry[b], tail_tile<A>(x, t - mem_tiles) * KT + b * 16, kNoPage);
      if (t + 4 < x.k1) look(t + 4);
      const char* p = kp + (col < 16 ? place[0].at : place[1].at) + (uint32_t)min(col & 15, col < 16 ? place[0].last : place[1].last) * (int64_t)rsb;
#pragma unroll
      for (int j = 0; j < D / 8; ++j) kr[j] = gload16(p + (j * 32 + half * 16));
    } else {
      const int key0 = (t - mem_tiles) * KT;
      const char* tile = kp + (int64_t)key0 * rsb;
      const uint32_t at = (uint32_t)min(col, nt - key0 - 1) * rsb + half * 16;
#pragma unroll
      for (int j = 0; j < D / 8; ++j) kr[j] = gload16(tile + (at + j * 32));
    }
    asm volatile("" ::: "memory");
  };
  const auto load_v = [&](int t) __attribute__((always_inline)) {
    if (t < mem_tiles) {
      const char* block = data + (int64_t)t * B::BYTES;
#pragma unroll
      for (int c = 0; c < NCT; ++c) {
        const uint4 w = gload16(block + (uint32_t)(B::V + (c * 32 + col) * 16));
        vr[c * 16] = w.x; vr[c * 16 + 1] = w.y; vr[c * 16 + 2] = w.z; vr[c * 16 + 3] = w.w;
        vb[c] = gload<uint8_t>(block + (uint32_t)B::v_scale(c * 32 + col));
      }
    } else if constexpr (A::kPaged) {                      // (of the tile that load_k went to last)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const char* p = vp + place[r >> 3].at;
        const uint32_t at = (uint32_t)min((r >> 2) % 2 * 8 + half * 4 + (r & 3), place[r >> 3].last) * rsb + col * 4;
#pragma unroll
        for (int c = 0; c < NCT; ++c) vr[c * 16 + r] = gload<uint32_t>(p + (at + c * 128));
      }
    } else {
      const int key0 = (t - mem_tiles) * KT;
      const char* tile = vp + (int64_t)key0 * rsb;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const uint32_t at = (uint32_t)min((r >> 2) * 8 + half * 4 + (r & 3), nt - key0 - 1) * rsb + col * 4;
#pragma unroll
        for (int c = 0; c < NCT; ++c) vr[c * 16 + r] = gload<uint32_t>(tile + (at + c * 128));
      }
    }
    asm volatile("" ::: "memory");
  };

  floatx16 o[NCT];
#pragma unroll
  for (int c = 0; c < NCT; ++c) o[c] = floatx16{};
  float m = -INFINITY, l = 0.0f;
  const auto step = [&](auto mem, int t) __attribute__((always_inline)) {
    floatx16 sc = floatx16{};
#pragma unroll
    for (int j = 0; j < D / 8; ++j) {
      floatx4 k;
      if constexpr (decltype(mem)::value)
        k = values4(j % 4 == 0 ? kr[j / 4].x : j % 4 == 1 ? kr[j / 4].y : j % 4 == 2 ? kr[j / 4].z : kr[j / 4].w, half, kb[j / 4]);
      else
        k = __builtin_bit_cast(floatx4, kr[j]);
#pragma unroll
      for (int e = 0; e < 4; ++e) sc = M::mma(k[e], q[j][e], sc);
    }
    uint32_t seen = ~0u;                                   // in pages: the tile's rows that the query sees
    if constexpr (A::kPaged && !decltype(mem)::value) {
      // Rows without a page were read from page 0, which may hold an infinity or NaN: their weights of 0 would not take
      // it away, and rows that see whole tiles are not formed again.
#pragma unroll
      for (int b = 0; b < 2; ++b)
        if (!place[b].there)
#pragma unroll
          for (int i = 0; i < 8 * NCT; ++i) vr[i / 8 * 16 + b * 8 + i % 8] = 0u;
      const int key0 = tail_tile<A>(x, t - mem_tiles) * KT;
      if (key0 < x.tail.all_from || key0 + KT > x.tail.all_to) seen = visible<uint32_t>(a, s, row, key0);
      if (!place[0].there) seen &= 0xFFFF0000u;
      if (!place[1].there) seen &= 0xFFFFu;
      seen >>= half * 4;
    }
    if (t + 4 < x.k1) load_k(t + 4);
    const int limit = (decltype(mem)::value ? nm - t * KT : row.seen - (t - mem_tiles) * KT) - half * 4;
    float top = -INFINITY;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const bool in = A::kPaged && !decltype(mem)::value ? (seen >> ((r >> 2) * 8 + (r & 3)) & 1u) != 0 : (r >> 2) * 8 + (r & 3) < limit;
      sc[r] = in ? sc[r] * s.scale_log2 : -INFINITY;
      top = fmaxf(top, sc[r]);
    }
    top = max32(top);
    if (__any(top > m + 8.0f)) {                           // (see attend_many)
      const float alpha = top > m + 8.0f ? exp2_(m - top) : 1.0f;
      m = top > m + 8.0f ? top : m;
      l *= alpha;
#pragma unroll
      for (int c = 0; c < NCT; ++c) o[c] *= alpha;
    }
    const float ref = m == -INFINITY ? 0.0f : m;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      sc[r] = exp2_(sc[r] - ref);
      l += sc[r];
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      floatx4 v[NCT];
#pragma unroll
      for (int c = 0; c < NCT; ++c) {
        if constexpr (decltype(mem)::value) v[c] = values4(vr[c * 16 + e], half, vb[c]);
        else
#pragma unroll
          for (int i = 0; i < 4; ++i) v[c][i] = __uint_as_float(vr[c * 16 + e * 4 + i]);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int c = 0; c < NCT; ++c) o[c] = M::mma(v[c][i], sc[e * 4 + i], o[c]);
    }
    if (t + 4 < x.k1) load_v(t + 4);
  };
  int t = x.k0 + wave;
  if (t < x.k1) {
    if (t >= mem_tiles) look(t);
    load_k(t);
    load_v(t);
  }
  for (; t < min(mem_tiles, x.k1); t += 4) step(std::true_type{}, t);
  for (; t < x.k1; t += 4) step(std::false_type{}, t);
  l += __shfl_xor(l, 32);

  // join the four wavefronts
  if (half == 0) ml[wave * R + col] = make_float2(m, l);
  __syncthreads();
  float top = -INFINITY;
#pragma unroll
  for (int w = 0; w < 4; ++w) top = fmaxf(top, ml[w * R + col].x);
  const float ref = top == -INFINITY ? 0.0f : top;
  const float mine = exp2_(m - ref);
  float total = 0.0f;
#pragma unroll
  for (int w = 0; w < 4; ++w) total += ml[w * R + col].y * exp2_(ml[w * R + col].x - ref);
#pragma unroll
  for (int c = 0; c < NCT; ++c)
#pragma unroll
    for (int e = 0; e < 4; ++e)
      *reinterpret_cast<floatx4*>(ob + (wave * R + col) * ROW + c * 32 + e * 8 + half * 4) =
          floatx4{o[c][4 * e], o[c][4 * e + 1], o[c][4 * e + 2], o[c][4 * e + 3]} * mine;
  if (wave == 0 && half == 0) joint->ml[col] = make_float2(top, total);
  finish<float, D, R, KT, ROW, 4>(a, s, x, ob, joint);
}

// ---------------------------------------------------------------------------
// fp32, many rows: 128 query rows to a unit, 32 to each wavefront, against key
// tiles of 64 rows (d = 128: 32) in two LDS stages.  The MFMA's rate bounds it:
// two workgroups to a CU, accumulators in the registers that the vector
// instructions use (256 of them: with more allowed, the compiler keeps
// accumulators apart and moves them), and vector instructions between MFMAs.
// 8 x 1600 queries of 16 heads of width 64 over 8256 rows 3390 us, 127 TFLOP/s
// of the 154 that a large product reaches; 2800 of 28 heads of width 128 over
// 8256 2500 us, 131.  With a workgroup to a CU and the moves 3756 and 2857.
// ---------------------------------------------------------------------------
template <int D>
struct F32Many {
  static constexpr int R = 128, KT = 4096 / D, WAVES = 4;
  static constexpr int TILE = KT * D;                      // elements of a K or V stage
  static constexpr int LDS = 4 * TILE * 4;                 // 64 KiB: two workgroups to a CU
  static constexpr int CPR = D / 4, COPIES = 4;            // 16-byte chunks per row, 1 KiB copies per wavefront
  __device__ static inline int k_chunk(int r, int c) { return c ^ (r & (CPR - 1)); }
};

template <int D, class A>
__global__ __launch_bounds__(256, 2) void attend_f32_many(A a) {
  using P = F32Many<D>;
  using M = Mfma<float>;
  using B = MemBlock<D>;
  constexpr int R = P::R, KT = P::KT, TILE = P::TILE, CPR = P::CPR, NCT = D / 32;
  constexpr int W = 2, TPR = 256 / KT, WPC = KT / 8;       // words of codes to a thread, threads to a key, words to a channel
  extern __shared__ __align__(16) char lds[];
  float* kbuf = reinterpret_cast<float*>(lds);             // [2][TILE]
  float* vbuf = kbuf + 2 * TILE;
  Unit x = unit_of<R, KT, 1>(a, blockIdx.x);
  const QuerySeq& s = a.seq[x.s];
  const int tid = threadIdx.x, lane = tid & 63, wave = wave_id(), half = lane >> 5, col = lane & 31;
  const Row row = row_of(a, s, x, x.rt * R + wave * 32 + col);
  const float* qp = static_cast<const float*>(s.q) + row.h * elems(s.q_hs, 4) + row.i * elems(s.q_rs, 4);
  uint32_t spare = kNoPage;                                // (see attend_many)
  Holes<KT, A> holes;
  if constexpr (A::kPaged) {
    if (s.nt > 0) spare = entry_of(a.pool, s, s.nt);
    holes.look(a, s, x);
  }
  floatx4 q[D / 8];                                        // channels 8 j + 4 half ..: one of each half to an MFMA
#pragma unroll
  for (int j = 0; j < D / 8; ++j) q[j] = row.live ? gload<floatx4>(qp + 8 * j + 4 * half) : floatx4{};
  floatx16 o[NCT];
#pragma unroll
  for (int c = 0; c < NCT; ++c) o[c] = floatx16{};
  float m = -INFINITY, l = 0.0f;

  uint32_t rsb = s.kv_rs * 16u;                            // row stride in bytes, below 2^24
  const char* kp = static_cast<const char*>(s.k) + x.g * ((int64_t)s.kv_hs * 16);
  const char* vp = static_cast<const char*>(s.v) + x.g * ((int64_t)s.kv_hs * 16);
  if constexpr (A::kPaged) {
    rsb = a.pool.row;
    kp = a.pool.k + x.g * a.pool.head;
    vp = a.pool.v + x.g * a.pool.head;
  }
  const char* data = s.mem + x.g * ((int64_t)s.mem_hs * 16);
  const int mem_tiles = x.mem_tiles, nt = s.nt, nm = s.nm;
  const int last_block = tiles_of<kMemRows>(nm) - 1;
  uint32_t entry[2] = {};                                  // in pages: of this wavefront's rows of the next tiles of V, K
  const auto group_key = [&](int t) __attribute__((always_inline)) {
    return tail_tile<A>(x, t - mem_tiles) * KT + wave * (KT / P::WAVES) / 16 * 16;
  };
  const auto copy = [&](const char* base, float* to, int t, bool is_k) __attribute__((always_inline)) {
    if constexpr (A::kPaged) {
      if (t == max(x.k0, mem_tiles)) entry[is_k] = entry_of(a.pool, s, group_key(t));
      const Place at = place_at(a.pool, s, entry[is_k], group_key(t), spare);
      if (t + 1 < x.k1) entry[is_k] = entry_of(a.pool, s, group_key(t + 1));
#pragma unroll
      for (int j = 0; j < P::COPIES; ++j) {
        const int J = wave * P::COPIES + j, r = (J * 64 + lane) / CPR, c = lane % CPR;
        dma16_opaque_s(base + at.at, (uint32_t)min(r & 15, at.last) * rsb + (is_k ? P::k_chunk(r, c) : c) * 16, to + J * 256);
      }
      return;
    }
    const int key0 = (t - mem_tiles) * KT, keys = nt - key0;
    const char* tile = base + (int64_t)key0 * rsb;
#pragma unroll
    for (int j = 0; j < P::COPIES; ++j) {
      const int J = wave * P::COPIES + j, r = (J * 64 + lane) / CPR, c = lane % CPR;
      dma16_opaque_s(tile, (uint32_t)min(r, keys - 1) * rsb + (is_k ? P::k_chunk(r, c) : c) * 16, to + J * 256);
    }
  };
  // a memory tile on its way: K by rows, V by channels
  uint32_t kw[W], vw[W], kb = 0, vb = 0;
  const int krow = tid / TPR, kw0 = tid % TPR * W, vch = tid * W / WPC, vw0 = tid * W % WPC;
  const auto fetch = [&](int t, int st) __attribute__((always_inline)) {
    if (t >= mem_tiles) {
      copy(kp, kbuf + st * TILE, t, true);
      copy(vp, vbuf + st * TILE, t, false);
      return;
    }
    const char* p = data + (int64_t)min(t * (KT / 32) + krow / 32, last_block) * B::BYTES;
    const char* v = data + (int64_t)min(t * (KT / 32) + vw0 / 4, last_block) * B::BYTES;
#pragma unroll
    for (int j = 0; j < W; ++j) {
      kw[j] = gload<uint32_t>(p + (krow & 31) * (D / 2) + (kw0 + j) * 4);
      vw[j] = gload<uint32_t>(v + B::V + vch * 16 + (vw0 % 4 + j) * 4);
    }
    kb = gload<uint8_t>(p + B::k_scale(krow & 31, kw0 / 4));
    vb = gload<uint8_t>(v + B::v_scale(vch));
  };
  const auto store = [&](int t, int st) __attribute__((always_inline)) {
    if (t >= mem_tiles) return;
    float* kd = kbuf + st * TILE + krow * D;
    float* vd = vbuf + st * TILE + vch;
#pragma unroll
    for (int j = 0; j < W; ++j) {
      float y[8];
      values8(kw[j], kb, y);
      const int c = (kw0 + j) * 2;
      *reinterpret_cast<floatx4*>(kd + P::k_chunk(krow, c) * 4) = floatx4{y[0], y[1], y[2], y[3]};
      *reinterpret_cast<floatx4*>(kd + P::k_chunk(krow, c + 1) * 4) = floatx4{y[4], y[5], y[6], y[7]};
      values8(vw[j], vb, y);
#pragma unroll
      for (int e = 0; e < 8; ++e) vd[((vw0 + j) * 8 + e) * D] = y[e];
    }
  };

  // (in pages) the rows of tile t that the lane's query sees
  const auto seen_of = [&](int t) __attribute__((always_inline)) {
    uint64_t bits = ~0ull;
    if constexpr (A::kPaged) {
      if (t < mem_tiles) return bits_below<uint64_t>(nm - t * KT);
      const int key0 = tail_tile<A>(x, t - mem_tiles) * KT;
      if (key0 < x.tail.all_from || key0 + KT > x.tail.all_to) bits = visible<uint64_t>(a, s, row, key0);
      if (x.holes) bits &= paged_bits<uint64_t>(a, s, key0);
    }
    return bits;
  };
  if (x.k0 < x.k1) {
    fetch(x.k0, 0);
    store(x.k0, 0);
  }
  dma_wait();
  __syncthreads();
  if constexpr (A::kPaged) x.holes = holes.found(a, s, x);
  for (int t = x.k0; t < x.k1; ++t) {
    const int st = (t - x.k0) & 1;
    if (t + 1 < x.k1) fetch(t + 1, st ^ 1);
    const int limit = (t < mem_tiles ? nm - t * KT : row.seen - (t - mem_tiles) * KT) - half * 4;
    bool masked;
    uint64_t seen = 0;
    if constexpr (A::kPaged) {
      seen = seen_of(t);
      masked = __any((seen & bits_below<uint64_t>(KT)) != bits_below<uint64_t>(KT));
      seen >>= half * 4;
    } else {
      masked = __any(limit <= KT - 5);                     // the tile's last key of this half is KT - 5 behind its first
    }
    const auto k_quad = [&](int b, int j) __attribute__((always_inline)) {
      return *reinterpret_cast<const floatx4*>(kbuf + st * TILE + (b * 32 + col) * D + P::k_chunk(b * 32 + col, 2 * j + half) * 4);
    };
    // (the key of accumulator register r of this half)
    const float* vd = vbuf + st * TILE + half * 4 * D + col;
    const auto v_one = [&](int b, int i) __attribute__((always_inline)) {
      const int r = i / NCT;
      return vd[(b * 32 + (r >> 2) * 8 + (r & 3)) * D + i % NCT * 32];
    };
    floatx16 sc[KT / 32];
    float ref;
    const auto scores = [&](int b, auto&& between) __attribute__((always_inline)) {
      floatx4 k[3] = {k_quad(b, 0), k_quad(b, 1), {}};
#pragma unroll
      for (int i = 0; i < D / 2; ++i) {
        if (i % 4 == 0 && i / 4 + 2 < D / 8) k[(i / 4 + 2) % 3] = k_quad(b, i / 4 + 2);
        sc[b] = M::mma(k[i / 4 % 3][i % 4], q[i / 4][i % 4], i ? sc[b] : floatx16{});
        pin(sc[b]);
        between(i);
      }
    };
    const auto reference = [&](float top) __attribute__((always_inline)) {
      top = max32(top);
      if (__any(top > m + 8.0f)) {                           // (see attend_many)
        const float alpha = top > m + 8.0f ? exp2_(m - top) : 1.0f;
        m = top > m + 8.0f ? top : m;
        l *= alpha;
#pragma unroll
        for (int c = 0; c < NCT; ++c) o[c] *= alpha;
      }
      ref = m == -INFINITY ? 0.0f : m;
    };
    const auto weight = [&](int b, int r) __attribute__((always_inline)) {
      sc[b][r] = exp2_(sc[b][r] - ref);
      l += sc[b][r];
      pin(l);
    };
    const auto values = [&](int b, auto&& between) __attribute__((always_inline)) {
      constexpr int N16 = 16 * NCT, AHEAD = 8;
      float v[AHEAD];
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) v[i] = v_one(b, i);
#pragma unroll
      for (int i = 0; i < N16; ++i) {
        o[i % NCT] = M::mma(v[i % AHEAD], sc[b][i / NCT], o[i % NCT]);
        pin(o[i % NCT]);
        if (i + AHEAD < N16) v[i % AHEAD] = v_one(b, i + AHEAD);
        between(i);
      }
    };
    const auto settle = [&](int b) __attribute__((always_inline)) {
      sc[b] *= s.scale_log2;
      if (!masked) return;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int j = b * 32 + (r >> 2) * 8 + (r & 3);
        if (A::kPaged ? (seen >> j & 1u) == 0 : j >= limit) sc[b][r] = -INFINITY;
      }
    };
    const auto all_weights = [&](int b) __attribute__((always_inline)) {
#pragma unroll
      for (int r = 0; r < 16; ++r) weight(b, r);
    };
    float top = -INFINITY;
    scores(0, [](int) {});
    settle(0);
#pragma unroll
    for (int r = 0; r < 16; ++r) top = fmaxf(top, sc[0][r]);
    reference(top);
    if constexpr (KT == 32) {
      all_weights(0);
      values(0, [](int) {});
    } else {                                               // vector instructions of a block between MFMAs of the other
      scores(1, [&](int i) __attribute__((always_inline)) {
#pragma unroll
        for (int r = i * 32 / D; r < (i + 1) * 32 / D; ++r) weight(0, r);
      });
      settle(1);
      top = -INFINITY;
      values(0, [&](int i) __attribute__((always_inline)) {
        if (i % NCT == 0) {
          top = fmaxf(top, sc[1][i / NCT]);
          pin(top);
        }
      });
      reference(top);
      all_weights(1);
      values(1, [](int) {});
    }
    if (t + 1 < x.k1) store(t + 1, st ^ 1);
    dma_wait();
    __syncthreads();
  }
  l += __shfl_xor(l, 32);
  write_rows<float, D, R>(a, s, x, row, wave * 32 + col, half, o, m, l);
  form_own<float, D, R, KT>(a, s, x, row, wave * 32, o, m, l);
}

// ---------------------------------------------------------------------------
// bf16, few rows (single tokens, short questions): 16 NR query rows to a unit.
// Its key tiles of 128 rows go round the wavefronts, each with sums of its own.
// A memory tile goes from HBM to registers and from there to the MFMAs: lane
// (i, g) = (lane % 16, lane / 16) reads a quarter of K row i of eight 16-row
// sets, and channel i's 32 rows of V block g, 16 bytes each; the sets are chosen
// (rows 4 T .. 4 T + 3 of each of the four blocks) so that set T's scores in
// lane (query, g) are those of V's rows 4 T .. of block g.  Memory bounds it on
// many long caches (32 tokens of 28 heads over up to 16384 rows, 164 MB, 39 us:
// 4.3 TB/s), its latency and the join on one (40256 rows, 22 MB: 13.5 us, 4.7 of
// them the join; 640 wavefronts wait 46% of their cycles and issue vector
// instructions in 32%) and on short ones (219 rows: 6 us).  Questions (7
// sequences, 180 rows of a head at most, 15.8 us) have one wavefront to a SIMD,
// which issues vector instructions, most of them to convert codes, in 38% of
// its cycles and waits in 41%.
// ---------------------------------------------------------------------------
template <int D, int NR, int KEYS = 128>                 // KEYS 32: without memories
struct Few {
  static constexpr int R = 16 * NR, KT = KEYS;
  static constexpr int WAVES = 4;
  static constexpr bool MEM = KEYS == 128;
  static constexpr int STEPS = D * NR == 256 ? 2 : 1;      // a memory tile's, by the registers of two wavefronts a SIMD
  static constexpr int OROW = D + 4;
  static constexpr int VBUF = 32 * D * 2;                  // bytes of a wavefront's tail V rows in LDS
  static constexpr int JOIN = WAVES * R * OROW * 4;
  static constexpr int STAT = WAVES * VBUF > JOIN ? WAVES * VBUF : JOIN;
  static constexpr int LDS = STAT + WAVES * R * 8 + (int)sizeof(Joint);
};
// 16-byte chunk of row r that holds its chunk c: the 8 rows that 32 lanes read
// 32 bytes each of lie in different banks.
template <int D>
__device__ inline int few_chunk(int r, int c) { return D == 128 ? c ^ ((r & 7) << 1) : c ^ (((r >> 1) & 3) << 1); }

template <int NR>
struct Stats {
  float m[NR], l[NR];
};
// Scores (log2 units) to weights against the running maximum; the factor that
// what was summed before has to be taken by.
template <int NR, int N>
__device__ inline void weigh(floatx4 (&sc)[NR][N], Stats<NR>& st, float (&alpha)[NR]) {
#pragma unroll
  for (int n = 0; n < NR; ++n) {
    float top = -INFINITY;
#pragma unroll
    for (int t = 0; t < N; ++t) top = fmaxf(fmaxf(fmaxf(top, sc[n][t][0]), fmaxf(sc[n][t][1], sc[n][t][2])), sc[n][t][3]);
    top = max32(max16(top));
    const float m2 = fmaxf(st.m[n], top), ref = m2 == -INFINITY ? 0.0f : m2;
    alpha[n] = exp2_(st.m[n] - ref);
    st.m[n] = m2;
    float sum = 0.0f;
#pragma unroll
    for (int t = 0; t < N; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        sc[n][t][r] = exp2_(sc[n][t][r] - ref);
        sum += sc[n][t][r];
      }
    st.l[n] = st.l[n] * alpha[n] + sum;
  }
}
// (rounded to bf16 for the second product, see Weights)
__device__ inline frag pack_weights(floatx4 x, floatx4 y) {
  return __builtin_bit_cast(frag, make_uint4(round2(x[0], x[1]), round2(x[2], x[3]), round2(y[0], y[1]), round2(y[2], y[3])));
}
__device__ inline uint32_t word(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }
__device__ inline float byte_scale(const uint2& v, int i) { return scale_of(((i < 4 ? v.x : v.y) >> (8 * (i & 3))) & 255u); }
template <int BYTES>
__device__ inline uint4 load_part(const char* p) {   // 16 or 8 bytes
  if constexpr (BYTES == 16) return gload16(p);
  const uint2 x = gload8(p);
  return make_uint4(x.x, x.y, 0, 0);
}

template <int D, int NR, class A, int KEYS = 128>
__global__ __launch_bounds__(256, 2) void attend_few(A a) {
  using P = Few<D, NR, KEYS>;
  using B = MemBlock<D>;
  constexpr int R = P::R, KT = P::KT, WAVES = P::WAVES, NS = D / 32, NC = D / 16, STEPS = P::STEPS, T = 8 / STEPS;
  extern __shared__ __align__(16) char lds[];
  const Unit x = unit_of<R, KT, WAVES>(a, blockIdx.x);
  const QuerySeq& s = a.seq[x.s];
  const int lane = threadIdx.x & 63, wave = wave_id(), g = lane >> 4, i16 = lane & 15;
  Row row[NR];
  const uint16_t* q[NR];
  frag qf[NR][NS];
  floatx4 o[NR][NC];
  Stats<NR> st;
#pragma unroll
  for (int n = 0; n < NR; ++n) {
    row[n] = row_of(a, s, x, x.rt * R + n * 16 + i16);
    q[n] = static_cast<const uint16_t*>(s.q) + row[n].h * elems(s.q_hs, 2) + row[n].i * elems(s.q_rs, 2);
    st.m[n] = -INFINITY;
    st.l[n] = 0.0f;
#pragma unroll
    for (int c = 0; c < NC; ++c) o[n][c] = floatx4{};
  }
  const float scale = s.scale_log2;
  int kti = x.k0 + wave;

  if (P::MEM && kti < min(x.k1, x.mem_tiles)) {
    // channels g D/4 .. of the queries, as the lanes hold K's
#pragma unroll
    for (int n = 0; n < NR; ++n)
#pragma unroll
      for (int j = 0; j < NS; ++j)
        qf[n][j] = row[n].live ? gload<frag>(q[n] + g * (D / 4) + j * 8) : frag{};
    const char* data = s.mem + x.g * ((int64_t)s.mem_hs * 16);
    const int last_block = tiles_of<kMemRows>(s.nm) - 1;
    uint4 kc[T], vc[NC];
    uint2 ks, vs;
    // step h of a tile: its 16-row sets T h .., and the rows of V that they are
    const auto load_k = [&](int t, int h) __attribute__((always_inline)) {
      const char* blk = data + (int64_t)min(t * 4 + (i16 >> 2), last_block) * B::BYTES;
#pragma unroll
      for (int j = 0; j < T; ++j) kc[j] = load_part<D / 8>(blk + ((h * T + j) * 4 + (i16 & 3)) * (D / 2) + g * (D / 8));
      ks = gload8(blk + B::k_scale(i16 & 3, g * (D / 4) / 32));
    };
    const auto load_v = [&](int t, int h) __attribute__((always_inline)) {
      const char* blk = data + (int64_t)min(t * 4 + g, last_block) * B::BYTES;
#pragma unroll
      for (int c = 0; c < NC; ++c) vc[c] = load_part<2 * T>(blk + B::V + (c * 16 + i16) * 16 + h * 2 * T);
      if constexpr (NC == 8) vs = gload8(blk + B::v_scale(i16));
      else vs = make_uint2(gload<uint32_t>(blk + B::v_scale(i16)), 0);
    };
    const int end = min(x.k1, x.mem_tiles);
    load_k(kti, 0);
    load_v(kti, 0);
    for (; kti < end; kti += WAVES) {
#pragma unroll
      for (int h = 0; h < STEPS; ++h) {
        const int next_t = h + 1 < STEPS ? kti : kti + WAVES, next_h = (h + 1) % STEPS;
        floatx4 sc[NR][T];
#pragma unroll
        for (int t = 0; t < T; ++t) {
#pragma unroll
          for (int n = 0; n < NR; ++n) sc[n][t] = floatx4{};
          const float ksc = byte_scale(ks, h * T + t);
#pragma unroll
          for (int j = 0; j < NS; ++j) {
            const frag kf = __builtin_bit_cast(frag, values8_bf16(word(kc[t], j), ksc));
#pragma unroll
            for (int n = 0; n < NR; ++n) sc[n][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[n][j], sc[n][t], 0, 0, 0);
          }
        }
        if (next_t < end) load_k(next_t, next_h);
        const int keys = s.nm - kti * KT;
#pragma unroll
        for (int n = 0; n < NR; ++n)
#pragma unroll
          for (int t = 0; t < T; ++t) sc[n][t] *= scale;
        if (keys < KT) {
#pragma unroll
          for (int n = 0; n < NR; ++n)
#pragma unroll
            for (int t = 0; t < T; ++t)
#pragma unroll
              for (int r = 0; r < 4; ++r)
                if (g * 32 + (h * T + t) * 4 + r >= keys) sc[n][t][r] = -INFINITY;
        }
        float alpha[NR];
        weigh<NR, T>(sc, st, alpha);
        frag pf[NR][T / 2];
#pragma unroll
        for (int n = 0; n < NR; ++n)
#pragma unroll
          for (int j = 0; j < T / 2; ++j) pf[n][j] = pack_weights(sc[n][2 * j], sc[n][2 * j + 1]);
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          const float vsc = byte_scale(vs, c);
#pragma unroll
          for (int n = 0; n < NR; ++n) o[n][c] *= alpha[n];
#pragma unroll
          for (int j = 0; j < T / 2; ++j) {
            const frag vf = __builtin_bit_cast(frag, values8_bf16(word(vc[c], j), vsc));
#pragma unroll
            for (int n = 0; n < NR; ++n) o[n][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[n][j], o[n][c], 0, 0, 0);
          }
        }
        if (next_t < end) load_v(next_t, next_h);
      }
    }
  }

  if (kti < x.k1) {
    // Tail rows, 32 at a time: K from HBM to registers, V through LDS, which
    // transposes 16-bit elements as they are read.
#pragma unroll
    for (int n = 0; n < NR; ++n)
#pragma unroll
      for (int j = 0; j < NS; ++j) qf[n][j] = row[n].live ? gload<frag>(q[n] + j * 32 + g * 8) : frag{};
    const int64_t rs = elems(s.kv_rs, 2);
    const uint16_t* kp = static_cast<const uint16_t*>(s.k) + x.g * elems(s.kv_hs, 2);
    const uint16_t* vp = static_cast<const uint16_t*>(s.v) + x.g * elems(s.kv_hs, 2);
    // In pages `key` counts the rows of the tiles that are taken; the rows 16 t .. of a step lie on one page, whose
    // entry is looked up a step ahead.
    uint32_t entry[2] = {};
    bool there[2] = {true, true};
    const auto at_row = [&](int key) __attribute__((always_inline)) {
      if constexpr (A::kPaged) return key + (key >= x.tail.sink_tiles * KT ? x.tail.skip * KT : 0);
      return key;
    };
    const auto look = [&](int key) __attribute__((always_inline)) {
      if constexpr (A::kPaged)
#pragma unroll
        for (int t = 0; t < 2; ++t) entry[t] = entry_of(a.pool, s, at_row(key) + t * 16);
    };
    uint16_t* vb = reinterpret_cast<uint16_t*>(lds + wave * P::VBUF);
    frag kc[2][NS];
    uint4 vc[NC];
    const auto load = [&](int key) {
      if constexpr (A::kPaged) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const int row0 = at_row(key) + t * 16;
          const Place at = place_at(a.pool, s, entry[t], row0, kNoPage);
          const char* kr = a.pool.k + x.g * a.pool.head + at.at;
          const char* vr = a.pool.v + x.g * a.pool.head + at.at;
          there[t] = at.there;
#pragma unroll
          for (int j = 0; j < NS; ++j) kc[t][j] = gload<frag>(kr + ((uint32_t)min(i16, at.last) * a.pool.row + (j * 32 + g * 8) * 2));
          const int rows = at.there ? s.nt - row0 : 0;
#pragma unroll
          for (int j = 0; j < NC / 2; ++j) {
            const int slot = j * 64 + lane, r = slot / (D / 8);
            vc[t * (NC / 2) + j] = r < rows ? gload16(vr + ((uint32_t)r * a.pool.row + slot % (D / 8) * 16)) : make_uint4(0, 0, 0, 0);
          }
        }
        return;
      }
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int j = 0; j < NS; ++j)
          kc[t][j] = gload<frag>(kp + min(key + t * 16 + i16, s.nt - 1) * rs + j * 32 + g * 8);
#pragma unroll
      for (int j = 0; j < NC; ++j) {
        const int slot = j * 64 + lane, t = slot / (D / 8);
        vc[j] = key + t < s.nt ? gload16(vp + (key + t) * rs + slot % (D / 8) * 8) : make_uint4(0, 0, 0, 0);
      }
    };
    // (each wavefront's 32-row steps: four to a key tile)
    const auto next = [&](int key) { return (key & (KT - 32)) != KT - 32 ? key + 32 : key + 32 + (WAVES - 1) * KT; };
    int end = min((x.k1 - x.mem_tiles) * KT, s.nt);
    if constexpr (A::kPaged) end = min((x.k1 - x.mem_tiles) * KT, s.nt - x.tail.skip * KT);
    int key = (kti - x.mem_tiles) * KT;
    if (key < end) {
      look(key);
      load(key);
      look(next(key));
    }
    while (key < end) {
#pragma unroll
      for (int j = 0; j < NC; ++j) {
        const int slot = j * 64 + lane, t = slot / (D / 8);
        *reinterpret_cast<uint4*>(vb + t * D + few_chunk<D>(t, slot % (D / 8)) * 8) = vc[j];
      }
      floatx4 sc[NR][2];
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int n = 0; n < NR; ++n) {
          sc[n][t] = floatx4{};
#pragma unroll
          for (int j = 0; j < NS; ++j) sc[n][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kc[t][j], qf[n][j], sc[n][t], 0, 0, 0);
        }
      const int here = at_row(key);
      const bool paged[2] = {there[0], there[1]};
      key = next(key);
      if (key < end) {
        load(key);
        look(next(key));
      }
      if constexpr (A::kPaged) {
        if (here >= x.tail.all_from && here + 32 <= x.tail.all_to && paged[0] && paged[1]) {
#pragma unroll
          for (int n = 0; n < NR; ++n)
#pragma unroll
            for (int t = 0; t < 2; ++t) sc[n][t] *= scale;
        } else {
          const uint32_t pages = (paged[0] ? 0xFFFFu : 0u) | (paged[1] ? 0xFFFF0000u : 0u);
#pragma unroll
          for (int n = 0; n < NR; ++n) {
            const uint32_t seen = (visible<uint32_t>(a, s, row[n], here) & pages) >> (g * 4);
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
              for (int r = 0; r < 4; ++r) sc[n][t][r] = seen >> (t * 16 + r) & 1u ? sc[n][t][r] * scale : -INFINITY;
          }
        }
      } else {
#pragma unroll
        for (int n = 0; n < NR; ++n)
#pragma unroll
          for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r)
              sc[n][t][r] = here + t * 16 + g * 4 + r < row[n].seen ? sc[n][t][r] * scale : -INFINITY;
      }
      float alpha[NR];
      weigh<NR, 2>(sc, st, alpha);
      frag pf[NR];
#pragma unroll
      for (int n = 0; n < NR; ++n) pf[n] = pack_weights(sc[n][0], sc[n][1]);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        s16x4 lo, hi;
        const int t = g * 4 + (i16 >> 2), ch = c * 16 + (i16 & 3) * 4;
        lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (__attribute__((address_space(3))) s16x4*)(vb + t * D + few_chunk<D>(t, ch >> 3) * 8 + (ch & 7)));
        hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (__attribute__((address_space(3))) s16x4*)(vb + (t + 16) * D + few_chunk<D>(t + 16, ch >> 3) * 8 + (ch & 7)));
        const uint2 x0 = __builtin_bit_cast(uint2, lo), x1 = __builtin_bit_cast(uint2, hi);
        const frag vf = __builtin_bit_cast(frag, make_uint4(x0.x, x0.y, x1.x, x1.y));
#pragma unroll
        for (int n = 0; n < NR; ++n) {
          o[n][c] *= alpha[n];
          o[n][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[n], o[n][c], 0, 0, 0);
        }
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
  }

  // join the wavefronts
  float2* ml = reinterpret_cast<float2*>(lds + P::STAT);              // [WAVES][R]
  Joint* joint = reinterpret_cast<Joint*>(ml + WAVES * R);
  float* ob = reinterpret_cast<float*>(lds);                          // [WAVES][R][OROW]
#pragma unroll
  for (int n = 0; n < NR; ++n) {
    st.l[n] += __shfl_xor(st.l[n], 16);
    st.l[n] += __shfl_xor(st.l[n], 32);
    if (g == 0) ml[wave * R + n * 16 + i16] = make_float2(st.m[n], st.l[n]);
  }
  __syncthreads();
#pragma unroll
  for (int n = 0; n < NR; ++n) {
    float top = -INFINITY, total = 0.0f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) top = fmaxf(top, ml[w * R + n * 16 + i16].x);
    const float ref = top == -INFINITY ? 0.0f : top, mine = exp2_(st.m[n] - ref);
#pragma unroll
    for (int w = 0; w < WAVES; ++w) total += ml[w * R + n * 16 + i16].y * exp2_(ml[w * R + n * 16 + i16].x - ref);
    if (wave == 0 && g == 0) joint->ml[n * 16 + i16] = make_float2(top, total);
#pragma unroll
    for (int c = 0; c < NC; ++c)
      *reinterpret_cast<floatx4*>(ob + (wave * R + n * 16 + i16) * P::OROW + c * 16 + g * 4) = o[n][c] * mine;
  }
  finish<uint16_t, D, R, KT, P::OROW, WAVES>(a, s, x, ob, joint);
}

// ---------------------------------------------------------------------------
// bf16, many rows (chunks): 256 query rows to a unit, 32 to each of eight
// wavefronts, against key tiles of 64 rows that they share in LDS, in four
// stages (with two, and a barrier every tile, 4096 queries of 28 heads over
// 20480 rows take 1067 us instead of 1051).  A step
// multiplies K of the next tile while it turns this tile's scores to weights,
// and then V of this tile: its MFMAs do not wait for its vector instructions.
// Tail rows are copied to LDS as they are, and V is transposed as it is read;
// a memory's codes go through registers, K as rows and V, whose codes lie by
// channel, as channels with their rows in the order that the weights have.
// ---------------------------------------------------------------------------
template <int D>
struct Many {
  static constexpr int R = 256, KT = 64, WAVES = 8;
  static constexpr int TILE = KT * D;                      // elements of a K or V stage
  static constexpr int LDS = 8 * TILE * 2;                 // four stages of K and of V
  static constexpr int CPR = D / 8;                        // 16-byte chunks per row
  static constexpr int COPIES = CPR / WAVES;               // 1 KiB copies of a tile per wavefront
  static constexpr int NKS = D / 16, NCT = D / 32;
  __device__ static inline int k_chunk(int r, int c) { return c ^ (r & (CPR - 1)); }
  __device__ static inline int v_chunk(int r, int c) { return D == 128 ? c ^ ((r & 3) << 2) : c ^ (((r >> 1) & 1) << 2); }
};

template <int D>
__device__ inline frag k_frag(const uint16_t* kd, int lane, int i) {   // i-th: keys i / NKS * 32 .., channels i % NKS * 16 ..
  using P = Many<D>;
  const int r = i / P::NKS * 32 + (lane & 31), c = 2 * (i % P::NKS) + (lane >> 5);
  return *reinterpret_cast<const frag*>(kd + r * D + P::k_chunk(r, c) * 8);
}
template <int D, bool MEM>
__device__ inline frag v_frag(const uint16_t* vd, int lane, int i) {   // i-th: keys i / NCT * 16 .., channels i % NCT * 32 ..
  using P = Many<D>;
  const int j = i / P::NCT, c = i % P::NCT, half = lane >> 5;
  if constexpr (MEM) {
    const int ch = c * 32 + (lane & 31);
    return *reinterpret_cast<const frag*>(vd + ch * P::KT + ((2 * j + half) ^ (ch & 7)) * 8);
  } else {
    typedef __attribute__((address_space(3))) s16x4 lds4;
    const int r = j * 16 + half * 4 + ((lane & 15) >> 2), ch = c * 32 + (lane & 16) + (lane & 3) * 4;
    const uint16_t* p = vd + r * D + P::v_chunk(r, ch >> 3) * 8 + (ch & 7);   // (row r + 8 has the same chunks)
    const uint2 x = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)p));
    const uint2 y = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(p + 8 * D)));
    return __builtin_bit_cast(frag, make_uint4(x.x, x.y, y.x, y.y));
  }
}

// Weights of the 16-key steps of a tile from their scores, one value at a time
// (value e of 32 is of step e / 8).  They are rounded to bf16 for the second
// product, half a step or 2^-8 of each at most, as its matrix cores have eight
// times the rate of fp32's; their sum takes them as they are.
struct Weights {
  uint32_t w[4][4];
  float even;
  __device__ __forceinline__ void value(int e, const floatx16 (&s)[2], float scale, float ref, float& l) {
    const float y = exp2_(__builtin_fmaf(s[e >> 4][e & 15], scale, -ref));
    l += y;
    pin(l);
    if (e & 1) {
      w[e >> 3][(e & 7) >> 1] = round2(even, y);
      pin(w[e >> 3][(e & 7) >> 1]);
    } else {
      even = y;
    }
  }
  __device__ inline frag step(int j) const { return __builtin_bit_cast(frag, make_uint4(w[j][0], w[j][1], w[j][2], w[j][3])); }
};

// One step: scores of the tile in kd into `next`, weights of the scores s and
// their products with the tile in vd (MEM: by channel) into o, and the largest
// next score (raw) of the lane.  The next tile's rows that the lane's query sees
// are `limit` first ones or (BITS) those of `seen`.  The order of MFMAs, LDS reads (kAhead
// fragments before their use) and vector instructions is that of the source.
constexpr int kAhead = 4;
template <int D, bool MEM, bool BITS>
__device__ __forceinline__ float many_step(const uint16_t* kd, const uint16_t* vd, int lane, const frag (&q)[D / 16], floatx16 (&s)[2],
                                  floatx16 (&next)[2], floatx16 (&o)[D / 32], float& l, float m, float scale, int limit, uint64_t seen,
                                  bool masked) {
  using P = Many<D>;
  constexpr int NK = 2 * P::NKS, NV = 4 * P::NCT;
  const float ref = m == -INFINITY ? 0.0f : m;
  Weights wt;
  frag f[kAhead + 1];
#pragma unroll
  for (int i = 0; i < kAhead; ++i) f[i] = k_frag<D>(kd, lane, i);
#pragma unroll
  for (int i = 0; i < NK; ++i) {
    if (i + kAhead < NK) f[(i + kAhead) % (kAhead + 1)] = k_frag<D>(kd, lane, i + kAhead);
    floatx16& x = next[i / P::NKS];
    x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[i % (kAhead + 1)], q[i % P::NKS], i % P::NKS ? x : floatx16{}, 0, 0, 0);
    pin(x);
#pragma unroll
    for (int e = 24 * i / NK; e < 24 * (i + 1) / NK; ++e) wt.value(e, s, scale, ref, l);
  }
#pragma unroll
  for (int i = 0; i < kAhead; ++i) f[i] = v_frag<D, MEM>(vd, lane, i);
  if (masked) {
    const int mine = limit - (lane >> 5) * 4;
    const uint64_t bits = seen >> ((lane >> 5) * 4);
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int j = b * 32 + (r >> 2) * 8 + (r & 3);
        if (BITS ? (bits >> j & 1u) == 0 : j >= mine) next[b][r] = -INFINITY;
      }
  }
  float top = -INFINITY;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    if (i + kAhead < NV) f[(i + kAhead) % (kAhead + 1)] = v_frag<D, MEM>(vd, lane, i + kAhead);
    floatx16& x = o[i % P::NCT];
    x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[i % (kAhead + 1)], wt.step(i / P::NCT), x, 0, 0, 0);
    pin(x);
    if (i < NV / 2) {
#pragma unroll
      for (int e = 24 + 16 * i / NV; e < 24 + 16 * (i + 1) / NV; ++e) wt.value(e, s, scale, ref, l);
    } else {
#pragma unroll
      for (int e = 32 * i / NV - 16; e < 32 * (i + 1) / NV - 16; ++e) {   // pairs of next scores
        top = fmaxf(fmaxf(top, next[0][e]), next[1][e]);
        pin(top);
      }
    }
  }
  return top;
}

template <int D, class A>
__global__ __launch_bounds__(512, 2) void attend_many(A a) {
  using P = Many<D>;
  using B = MemBlock<D>;
  constexpr int R = P::R, KT = P::KT, TILE = P::TILE, CPR = P::CPR, NKS = P::NKS, NCT = P::NCT;
  constexpr int W = D / 64;                                // code words per thread and operand of a memory tile
  extern __shared__ __align__(16) char lds[];
  uint16_t* kbuf = reinterpret_cast<uint16_t*>(lds);       // [4][TILE]
  uint16_t* vbuf = kbuf + 4 * TILE;
  Unit x = unit_of<R, KT, 1>(a, blockIdx.x);
  const QuerySeq& s = a.seq[x.s];
  const int tid = threadIdx.x, lane = tid & 63, wave = wave_id(), half = lane >> 5, col = lane & 31;
  const float scale = fabsf(s.scale_log2);
  const Row row = row_of(a, s, x, x.rt * R + wave * 32 + col);
  uint32_t spare = kNoPage;                                // of the rows that are read where there is no page
  Holes<KT, A> holes;
  if constexpr (A::kPaged) {
    // (values without a page are multiplied by weights of 0: finite ones, as the last row's are but for those that see it)
    if (s.nt > 0) spare = entry_of(a.pool, s, s.nt);
    holes.look(a, s, x);
  }
  frag q[NKS];
  {
    const uint16_t* p = static_cast<const uint16_t*>(s.q) + row.h * elems(s.q_hs, 2) + row.i * elems(s.q_rs, 2);
    const uint32_t flip = s.scale_log2 < 0.0f ? 0x80008000u : 0u;   // (a negative scale goes into the queries' signs)
#pragma unroll
    for (int j = 0; j < NKS; ++j) {
      uint4 w = row.live ? gload16(p + j * 16 + half * 8) : make_uint4(0, 0, 0, 0);
      w.x ^= flip; w.y ^= flip; w.z ^= flip; w.w ^= flip;
      q[j] = __builtin_bit_cast(frag, w);
    }
  }
  floatx16 o[NCT];
#pragma unroll
  for (int c = 0; c < NCT; ++c) o[c] = floatx16{};
  float m = -INFINITY, l = 0.0f;                           // reference of the sums (log2 units), sum of weights

  uint32_t rsb = s.kv_rs * 16u;                            // row stride in bytes, below 2^24
  const char* kp = static_cast<const char*>(s.k) + x.g * ((int64_t)s.kv_hs * 16);
  const char* vp = static_cast<const char*>(s.v) + x.g * ((int64_t)s.kv_hs * 16);
  if constexpr (A::kPaged) {
    rsb = a.pool.row;
    kp = a.pool.k + x.g * a.pool.head;
    vp = a.pool.v + x.g * a.pool.head;
  }
  const char* data = s.mem + x.g * ((int64_t)s.mem_hs * 16);
  const int mem_tiles = x.mem_tiles, nt = s.nt, nm = s.nm;
  const int last_block = tiles_of<kMemRows>(nm) - 1;
  // tail copies: lane / CPR is the row of a copy's 64 / CPR rows, lane % CPR its chunk
  const uint32_t lane_row = lane / CPR, lane_off = lane_row * rsb;
  uint32_t entry[2] = {};                                  // in pages: of this wavefront's rows of the next tiles of V, K
  const auto group_key = [&](int t) __attribute__((always_inline)) { return tail_tile<A>(x, t - mem_tiles) * KT + wave / 2 * 16; };
  const auto copy = [&](const char* base, uint16_t* to, int t, bool is_k) __attribute__((always_inline)) {
    if constexpr (A::kPaged) {
      if (t == max(x.k0, mem_tiles)) entry[is_k] = entry_of(a.pool, s, group_key(t));
      const Place at = place_at(a.pool, s, entry[is_k], group_key(t), spare);
      if (t + 1 < x.k1) entry[is_k] = entry_of(a.pool, s, group_key(t + 1));
#pragma unroll
      for (int j = 0; j < P::COPIES; ++j) {
        const int J = wave * P::COPIES + j, r = J * (64 / CPR) + lane_row, c = lane % CPR;
        const uint32_t chunk = (is_k ? P::k_chunk(r, c) : P::v_chunk(r, c)) * 16;
        dma16_opaque_s(base + at.at, (uint32_t)min(r & 15, at.last) * rsb + chunk, to + J * 512);
      }
      return;
    }
    const int key0 = (t - mem_tiles) * KT, keys = nt - key0;
    const char* tile = base + (int64_t)key0 * rsb;
#pragma unroll
    for (int j = 0; j < P::COPIES; ++j) {
      const int J = wave * P::COPIES + j, r0 = J * (64 / CPR), r = r0 + lane_row, c = lane % CPR;
      const uint32_t chunk = (is_k ? P::k_chunk(r, c) : P::v_chunk(r, c)) * 16;
      if (keys >= KT) dma16_opaque_s(tile + (int64_t)r0 * rsb, lane_off + chunk, to + J * 512);
      else dma16_opaque_s(tile, (uint32_t)min(r, keys - 1) * rsb + chunk, to + J * 512);
    }
  };
  // a memory tile on its way: K by rows, 8 threads to one; V by channels, 8 / W threads to one
  uint32_t kw[W], vw[W], kb = 0, vb = 0;
  const int krow = tid / 8, vch = tid * W / 8, vt8 = tid * W % 8;
  const auto words = [&](const char* p, uint32_t (&w)[W]) __attribute__((always_inline)) {
    if constexpr (W == 2) {
      const uint2 y = gload8(p);
      w[0] = y.x; w[1] = y.y;
    } else {
      w[0] = gload<uint32_t>(p);
    }
  };
  const auto fetch_k = [&](int t, int st) __attribute__((always_inline)) {
    if (t >= mem_tiles) { copy(kp, kbuf + st * TILE, t, true); return; }
    const char* p = data + (int64_t)min(t * 2 + wave / 4, last_block) * B::BYTES;   // (wavefronts 4 .. have rows 32 ..)
    words(p + (uint32_t)((krow & 31) * (D / 2) + (tid & 7) * (D / 16)), kw);
    kb = gload<uint8_t>(p + (uint32_t)B::k_scale(krow & 31, (tid & 7) * (D / 8) / 32));
  };
  const auto fetch_v = [&](int t, int st) __attribute__((always_inline)) {
    if (t >= mem_tiles) { copy(vp, vbuf + st * TILE, t, false); return; }
    const char* p = data + (int64_t)(t * 2) * B::BYTES;
    const uint32_t block = vt8 >= 4 && t * 2 < last_block ? B::BYTES : 0;
    words(p + (block + (uint32_t)(B::V + vch * 16 + vt8 % 4 * 4)), vw);
    vb = gload<uint8_t>(p + (block + (uint32_t)B::v_scale(vch)));
  };
  const auto store_k = [&](int t, int st) __attribute__((always_inline)) {
    if (t >= mem_tiles) return;
    uint16_t* p = kbuf + st * TILE + krow * D;
#pragma unroll
    for (int j = 0; j < W; ++j)
      *reinterpret_cast<uint4*>(p + P::k_chunk(krow, (tid & 7) * W + j) * 8) = values8_bf16(kw[j], scale_of(kb));
  };
  const auto store_v = [&](int t, int st) __attribute__((always_inline)) {
    if (t >= mem_tiles) return;
#pragma unroll
    for (int j = 0; j < W; ++j) {
      const uint4 y = values8_bf16(vw[j], scale_of(vb));
      const int t8 = vt8 + j, c = t8 >> 1 << 1;            // rows 8 t8 .. of the tile, in the 16-row step t8 / 2
      uint16_t* p = vbuf + st * TILE + vch * KT + (t8 & 1) * 4;
      *reinterpret_cast<uint2*>(p + (c ^ (vch & 7)) * 8) = make_uint2(y.x, y.y);
      *reinterpret_cast<uint2*>(p + ((c + 1) ^ (vch & 7)) * 8) = make_uint2(y.z, y.w);
    }
  };
  const auto limit_of = [&](int t) __attribute__((always_inline)) {                       // keys of tile t that the lane's query sees
    return t < mem_tiles ? nm - t * KT : row.seen - (t - mem_tiles) * KT;
  };
  const auto seen_of = [&](int t) __attribute__((always_inline)) {                        // in pages: a bit each
    uint64_t bits = ~0ull;
    if constexpr (A::kPaged) {
      if (t < mem_tiles) return bits_below<uint64_t>(nm - t * KT);
      const int key0 = tail_tile<A>(x, t - mem_tiles) * KT;
      if (key0 < x.tail.all_from || key0 + KT > x.tail.all_to) bits = visible<uint64_t>(a, s, row, key0);
      if (x.holes) bits &= paged_bits<uint64_t>(a, s, key0);
    }
    return bits;
  };
  const auto raise = [&](float top) __attribute__((always_inline)) {                      // largest raw score of the tile to come
    top = max32(top) * scale;
    // A row's sums keep their reference until one of its scores passes it by 8: weights stay below 2^8, few tiles scale
    // O, and what a wavefront's other rows see has no part in it.
    if (__any(top > m + 8.0f)) {
      const float alpha = top > m + 8.0f ? exp2_(m - top) : 1.0f;
      m = top > m + 8.0f ? top : m;
      l *= alpha;
#pragma unroll
      for (int c = 0; c < NCT; ++c) o[c] *= alpha;
    }
  };

  if (x.k0 < x.k1) {
    floatx16 s0[2], s1[2];
    const auto first = [&](int stage) __attribute__((always_inline)) {       // scores of the first tile
      if constexpr (A::kPaged) x.holes = holes.found(a, s, x);
      const uint16_t* kd = kbuf + stage * TILE;
      s0[0] = s0[1] = floatx16{};
#pragma unroll
      for (int i = 0; i < 2 * NKS; ++i)
        s0[i / NKS] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k_frag<D>(kd, lane, i), q[i % NKS], s0[i / NKS], 0, 0, 0);
      const int mine = limit_of(x.k0) - half * 4;
      const uint64_t bits = seen_of(x.k0) >> (half * 4);
      float top = -INFINITY;
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int j = b * 32 + (r >> 2) * 8 + (r & 3);
          if (A::kPaged ? (bits >> j & 1u) == 0 : j >= mine) s0[b][r] = -INFINITY;
          top = fmaxf(top, s0[b][r]);
        }
      raise(top);
    };
    const auto step = [&](auto mem, auto swapped, int t, int kst, int vst) __attribute__((always_inline)) {
      floatx16(&sc)[2] = decltype(swapped)::value ? s1 : s0;
      floatx16(&next)[2] = decltype(swapped)::value ? s0 : s1;
      const int limit = limit_of(t + 1);
      const uint64_t seen = A::kPaged && t + 1 < x.k1 ? seen_of(t + 1) : ~0ull;
      const bool masked = A::kPaged ? __any(seen != ~0ull) : __any(limit < KT);
      const float top = many_step<D, decltype(mem)::value, A::kPaged>(kbuf + kst * TILE, vbuf + vst * TILE, lane, q, sc, next, o, l, m,
                                                                      scale, limit, seen, masked);
      if (t + 1 < x.k1) raise(top);
    };
    const auto keep = [&]() __attribute__((always_inline)) {
      s0[0] = s1[0];
      s0[1] = s1[1];
    };
    const auto barrier = []() __attribute__((always_inline)) {
      dma_wait();
      __syncthreads();
    };
    chunk_steps(x.k0, x.k1, min(max(mem_tiles, x.k0), x.k1), fetch_k, fetch_v, store_k, store_v, first, step, keep, barrier);
  }
  l += __shfl_xor(l, 32);
  write_rows<uint16_t, D, R>(a, s, x, row, wave * 32 + col, half, o, m, l);
  form_own<uint16_t, D, R, KT>(a, s, x, row, wave * 32, o, m, l);
}

// ---------------------------------------------------------------------------
// Puts the partial results of query rows' splits together.  SHARES threads to a
// row and 4 channels: one for up to 8 splits (it has all its loads on their way
// at once), 4 for more, a workgroup of 1024 threads for many splits of few rows.
// ---------------------------------------------------------------------------
struct JoinTile {
  int s, g, rt, splits;
  int64_t slot;
};
template <class A>
__device__ inline JoinTile split_tile(const A& a, int j) {   // the j-th row tile with splits
  const int lane = threadIdx.x & 63;
  JoinTile x;
  int tile;
  if (a.whole > 0) {
    tile = a.whole + j;
    x.s = seq_of(a.unit0, a.n_seqs, tile);
    tile -= a.unit0[x.s];
    x.slot = (int64_t)j * a.seq[0].splits;
  } else {
    int first = lane < A::kSeqs && lane < a.n_seqs && a.seq[lane].splits > 1 ? a.h_kv * a.seq[lane].row_tiles : 0;
    const int count = first;
    for (int k = 1; k < A::kSeqs; k *= 2) {
      const int y = __shfl_up(first, k);
      if (lane >= k) first += y;
    }
    first -= count;                              // split row tiles of the sequences before
    const uint64_t at = __ballot(count > 0 && first <= j);
    x.s = uniform(63 - __clzll((long long)at));
    tile = j - uniform(__shfl(first, x.s));
    x.slot = a.seq[x.s].slot0 + (int64_t)tile * a.seq[x.s].splits;
  }
  const QuerySeq& s = a.seq[x.s];
  x.splits = s.splits;
  x.rt = s.row_tiles - 1 - tile / a.h_kv;
  x.g = tile % a.h_kv;
  return x;
}

template <typename T, int D, int R, int SHARES, int THREADS, class A>
__global__ __launch_bounds__(THREADS) void join_splits(A a) {
  constexpr int TPR = D / 4, ROWS = THREADS / TPR / SHARES; // rows per workgroup
  constexpr int E = (int)sizeof(T);
  const JoinTile x = split_tile(a, blockIdx.x);
  const QuerySeq& s = a.seq[x.s];
  const int c = threadIdx.x % TPR * 4, share = threadIdx.x / TPR % SHARES, r = blockIdx.y * ROWS + threadIdx.x / TPR / SHARES;
  const int row = x.rt * R + r;
  const bool live = row < a.group * s.nq;
  if (__syncthreads_or(live) == 0) return;
  const float2* ml = a.part_ml + x.slot * R + r;
  const float* po = a.part_o + (x.slot * R + r) * D + c;
  float m = -INFINITY, l = 0.0f;
  floatx4 o = floatx4{};
  if (live) {
#pragma unroll 4
    for (int p = share; p < x.splits; p += SHARES) {
      const floatx2 y = gload<floatx2>(ml + (int64_t)p * R);
      const floatx4 z = gload<floatx4>(po + (int64_t)p * R * D);
      const float m2 = fmaxf(m, y[0]), ref = m2 == -INFINITY ? 0.0f : m2;
      const float was = exp2_(m - ref), is = exp2_(y[0] - ref);
      l = l * was + y[1] * is;
      o = o * was + z * is;
      m = m2;
    }
  }
  if constexpr (SHARES > 1) {
    __shared__ floatx4 os[THREADS];
    __shared__ float2 mls[THREADS];
    os[threadIdx.x] = o;
    mls[threadIdx.x] = make_float2(m, l);
    __syncthreads();
    if (share != 0) return;
    float top = -INFINITY;
#pragma unroll
    for (int p = 0; p < SHARES; ++p) top = fmaxf(top, mls[threadIdx.x + p * TPR].x);
    const float ref = top == -INFINITY ? 0.0f : top;
    o = floatx4{};
    l = 0.0f;
#pragma unroll
    for (int p = 0; p < SHARES; ++p) {
      const float w = exp2_(mls[threadIdx.x + p * TPR].x - ref);
      l += mls[threadIdx.x + p * TPR].y * w;
      o += os[threadIdx.x + p * TPR] * w;
    }
    m = top;
  }
  if (!live) return;
  const int i = row / a.group, h = x.g * a.group + row % a.group;
  put4(static_cast<T*>(s.out) + h * elems(s.out_hs, E) + i * elems(s.out_rs, E) + c, over(o, l));
  if (c == 0 && s.lse) s.lse[h * (int64_t)s.lse_hs + i] = log_of(m, l);
}

// ---------------------------------------------------------------------------
// Plans and launches.
// ---------------------------------------------------------------------------
// Tail rows that a row tile of R rows takes, about.
template <int R, class A>
inline int tail_rows(const A& a, const QuerySeq& s) {
  if constexpr (A::kPaged) return (int)std::min<int64_t>(s.nt, (int64_t)a.sinks + a.window + std::min(s.nq, R / a.group));
  return s.nt;
}

template <int R, int D>
constexpr int64_t partials() { return kPartBytes / (R * (D * 4 + 8)); }

template <int R, int KT, class A>
int64_t count_tiles(A& a, int64_t* keys) {
  int64_t n = 0;
  *keys = 0;
  for (int i = 0; i < a.n_seqs; ++i) {
    QuerySeq& s = a.seq[i];
    s.row_tiles = (int)(((int64_t)a.group * s.nq + R - 1) / R);
    n += (int64_t)a.h_kv * s.row_tiles;
    *keys += (int64_t)a.h_kv * s.row_tiles * (tiles_of<KT>(s.nm) + tiles_of<KT>(tail_rows<R>(a, s)));
  }
  return n;
}

// Few rows: key tiles in shares of a multiple of kFewWaves, the same number to
// each of a workgroup's wavefronts.  A compute unit has its workgroups side by
// side, so a call takes as long as the fullest one: for each of some k the
// smallest shares of which a compute unit has at most k, and of those the ones
// with the least key tiles on the fullest, k - 1 average shares and the largest
// one, and 6 tiles' time to begin and end each.  us, with these and with shares
// of the keys over three times the compute units: 32 tokens over 200 to 16384
// rows 33 and 37, over 16384 50 and 56, 8 over up to 8192 11.5 and 13.4, 100 over
// up to 8000 73 and 90, 7 prompts of 45 over up to 4096 (width 64) 16 and 20.
struct Shares {
  int64_t units = 0, parts = 0, tiles = 0, largest = 0;
};
template <int R, int KT, class A>
Shares set_shares(A& a, int64_t share) {
  Shares x;
  for (int i = 0; i < a.n_seqs; ++i) {
    QuerySeq& s = a.seq[i];
    const int64_t t = std::max(tiles_of<KT>(s.nm) + tiles_of<KT>(tail_rows<R>(a, s)), 1), heads = (int64_t)a.h_kv * s.row_tiles;
    s.splits = (int)((t + share - 1) / share);
    a.unit0[i] = (int)x.units;
    s.slot0 = (int)x.parts;
    x.units += heads * s.splits;
    if (s.splits > 1) x.parts += heads * s.splits;
    x.tiles += heads * t;
    x.largest = std::max(x.largest, (t + s.splits - 1) / s.splits);
    if (x.units > INT32_MAX) break;
  }
  return x;
}
// Short key tiles, of 32 rows (bf16 in pages without memories), count a quarter of those of 128,
// and no split and what a join costs are weighed too: in tiles' time 5 and 5 for
// each partial on a compute unit (32 rows: 8 and 12).  us, split and not, width
// 128, 4 KV heads: a token that sees 1028 rows 9.0 and 14.1, 516 7.9 and 9.7, 132 7.7
// and 6.7; 16 tokens that see 516 11.2 and 12.6, 32 13.8 and 12.9; trees over 500
// rows, 112 rows of a head 11.2 and 12.7, four of 448 16.0 and 13.2.
template <int R, int KT, bool kShort, class A>
bool plan_shares(A& a, int64_t slots, int cus) {
  constexpr int kEnds = kShort ? 24 : 6;
  const auto join = [cus](const Shares& x) { return x.parts == 0 ? 0.0 : R == 16 ? 5 + 5.0 * x.parts / cus : 8 + 12.0 * x.parts / cus; };

  int64_t keys, most = 1;
  count_tiles<R, KT>(a, &keys);
  a.whole = 0;
  for (int i = 0; i < a.n_seqs; ++i) most = std::max(most, (int64_t)tiles_of<KT>(a.seq[i].nm) + tiles_of<KT>(tail_rows<R>(a, a.seq[i])));
  int64_t best = (most + kFewWaves - 1) / kFewWaves, high = best;   // in kFewWaves tiles: no split
  double least = 1e30;
  if constexpr (kShort) {
    const Shares x = set_shares<R, KT>(a, high * kFewWaves);
    const double n = (double)((x.units + cus - 1) / cus);
    least = (n - 1) * x.tiles / x.units + x.largest + kEnds * n;
  }
  for (int k : {1, 2, 3, 4, 6, 8}) {
    int64_t low = 1;
    if (set_shares<R, KT>(a, high * kFewWaves).units > (int64_t)k * cus) continue;
    while (low < high) {
      const int64_t mid = (low + high) / 2;
      if (set_shares<R, KT>(a, mid * kFewWaves).units <= (int64_t)k * cus) high = mid; else low = mid + 1;
    }
    const Shares x = set_shares<R, KT>(a, high * kFewWaves);
    const double n = (double)((x.units + cus - 1) / cus), cost = (n - 1) * x.tiles / x.units + x.largest + kEnds * n + (kShort ? join(x) : 0);
    if (x.parts <= slots && cost < least) {
      least = cost;
      best = high;
    }
    if (high == 1) break;
  }
  const Shares x = set_shares<R, KT>(a, best * kFewWaves);
  a.units = (int)x.units;
  return x.units <= INT32_MAX;
}

// As many whole row tiles as fill the chip a number of times, and the rest in
// so many shares that it takes least: rounds of a share's key tiles and `ends`
// more to begin and end it, and the join, about as much again to launch and
// `partial` for each, in key tiles' time (bf16 about 1.7 us, fp32 4 us).
template <int R, int KT, class A>
int64_t plan_rounds(A& a, int64_t slots, int width, double ends, double partial) {
  int64_t keys;
  const int64_t n = count_tiles<R, KT>(a, &keys);
  if (n > INT32_MAX / 64) return -1;
  const int64_t whole = n / width * width, rest = n - whole;
  int splits = 1;
  if (rest > 0) {
    const double tiles = (double)keys / n;
    const int64_t most = std::max<int64_t>(1, std::min<int64_t>(slots / rest, 512));
    double best = 1e30;
    for (int c = 1; c <= most && c <= tiles; ++c) {
      const double cost = (double)((rest * c + width - 1) / width) * (tiles / c + ends) + (c > 1 ? ends + partial * rest * c : 0);
      if (cost < best) { best = cost; splits = c; }
    }
  }
  a.whole = (int)(splits == 1 ? n : whole);
  int64_t units = 0, parts = 0;
  for (int i = 0; i < a.n_seqs; ++i) {
    QuerySeq& s = a.seq[i];
    s.splits = splits;
    a.unit0[i] = (int)units;
    s.slot0 = (int)parts;
    const int64_t u = (int64_t)a.h_kv * s.row_tiles * (a.whole > 0 ? 1 : splits);
    units += u;
    parts += u;
  }
  a.units = (int)(splits == 1 ? n : whole + rest * splits);
  return splits == 1 ? 0 : rest;
}

// Sequences of different lengths, of which plan_rounds' equal splits would let
// the longest end last: shares of the same number of key tiles, all row tiles in
// their order, the number of them that takes least.  `width` units at a time
// take as long as the longest share, more of them their average and half a share
// to end.
template <int R, int KT, class A>
int64_t plan_lengths(A& a, int64_t slots, int width, double ends, double partial) {
  int64_t most = 1;
  for (int i = 0; i < a.n_seqs; ++i) most = std::max(most, (int64_t)tiles_of<KT>(a.seq[i].nm) + tiles_of<KT>(tail_rows<R>(a, a.seq[i])));
  int64_t best = most;
  double least = 1e30;
  for (int64_t share = most;;) {
    const Shares x = set_shares<R, KT>(a, share);
    if (x.parts > slots || x.units > INT32_MAX) break;
    const double whole = x.largest + ends, all = (x.tiles + ends * x.units) / width;
    const double cost = (x.units <= width ? whole : all + whole / 2) + (x.parts > 0 ? ends + partial * x.parts : 0);
    if (cost < least) {
      least = cost;
      best = share;
    }
    if (share == 1) break;
    share = std::max<int64_t>(1, share - (share + 7) / 8);
  }
  a.whole = 0;
  a.units = (int)set_shares<R, KT>(a, best).units;
  int64_t joins = 0;
  for (int i = 0; i < a.n_seqs; ++i)
    if (a.seq[i].splits > 1) joins += (int64_t)a.h_kv * a.seq[i].row_tiles;
  return joins;
}

// The arguments with room for one sequence.
inline void first_of(const AttendArgs<kQueriesPerLaunch>& a, AttendArgs<1>& x) {
  x.seq[0] = a.seq[0];
  x.unit0[0] = a.unit0[0];
  x.n_seqs = 1; x.h_kv = a.h_kv; x.group = a.group; x.causal = a.causal; x.whole = a.whole; x.units = a.units;
  x.part_o = a.part_o; x.part_ml = a.part_ml; x.arrived = a.arrived; x.joined = a.joined;
}
inline void first_of(const PagedArgs<kQueriesPerLaunch>& a, PagedArgs<1>& x) {
  first_of(static_cast<const AttendArgs<kQueriesPerLaunch>&>(a), static_cast<AttendArgs<1>&>(x));
  x.pool = a.pool; x.window = a.window; x.sinks = a.sinks;
}
// The join of the split row tiles.
template <typename T, int D, int R, int SHARES, int THREADS, class A>
void join(const A& a, int64_t joins, hipStream_t st) {
  constexpr int ROWS = THREADS / (D / 4) / SHARES;
  join_splits<T, D, R, SHARES, THREADS, A><<<dim3((unsigned)joins, R / ROWS), THREADS, 0, st>>>(a);
}
template <typename T, typename P, int D, class A, typename Kernel>
hipError_t launch(const A& a, int64_t joins, int splits, Kernel kernel, hipStream_t st) {
  kernel<<<a.units, 64 * P::WAVES, P::LDS, st>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || joins == 0) return e;
  if (splits <= 8) join<T, D, P::R, 1, 256>(a, joins, st);
  else if (splits <= 32 || P::R >= 128) join<T, D, P::R, 4, 256>(a, joins, st);
  else if constexpr (P::R < 128) join<T, D, P::R, 1024 / (D / 4), 1024>(a, joins, st);
  return hipGetLastError();
}
template <typename T, typename P, int D, class A, typename One, typename All>
hipError_t launch(A& a, void* ws, int64_t joins, int splits, One one, All all, hipStream_t st) {
  a.part_o = static_cast<float*>(ws);
  a.part_ml = reinterpret_cast<float2*>(a.part_o + partials<P::R, D>() * P::R * D);
  a.arrived = reinterpret_cast<int*>(static_cast<char*>(ws) + kPartBytes);
  if (a.n_seqs > 1) return launch<T, P, D>(a, joins, splits, all, st);
  typename A::One x;
  first_of(a, x);
  return launch<T, P, D>(x, joins, splits, one, st);
}

// Few rows, in shares of at least a key tile for each wavefront.  Units join
// themselves where that takes one of them `kJoinBatches` rounds of loads at
// most (its threads have 8 partials of 4 channels on their way each); past
// that a kernel for it is as fast or faster.  us, with the kernel and without:
// a row of 7 heads over 1024 keys of width 128 (1 round) 10.8 and 8.7, of 4
// heads over 32768 keys of width 64 (3) 12.8 and 10.7; 42 rows over 1024 keys
// of width 128 (4) 13.7 and 15.6.
constexpr int kJoinBatches = 3;
template <typename T, typename P, int D, class A, typename One, typename All>
hipError_t launch_shares(A& a, void* ws, int cus, One one, All all, hipStream_t st) {
  constexpr int64_t slots = partials<P::R, D>();
  static_assert(slots <= kMaxPartials, "a counter to a partial");
  static_assert(P::WAVES == kFewWaves, "shares for the workgroup's wavefronts");
  if (!plan_shares<P::R, P::KT, sizeof(T) == 2 && P::KT == 32>(a, slots, cus)) return hipErrorInvalidConfiguration;
  int splits = 1;
  int64_t joins = 0, batches = 0;
  for (int i = 0; i < a.n_seqs; ++i) {
    const QuerySeq& s = a.seq[i];
    if (s.splits == 1) continue;
    const int64_t items = std::min<int64_t>(P::R, (int64_t)a.group * s.nq) * (D / 4), threads = 64 * P::WAVES;
    const int64_t passes = (items + threads - 1) / threads, shares = std::max<int64_t>(1, threads / items);
    joins += (int64_t)a.h_kv * s.row_tiles;
    splits = std::max(splits, s.splits);
    batches = std::max(batches, passes * ((s.splits + 8 * shares - 1) / (8 * shares)));
  }
  a.joined = batches <= kJoinBatches;
  return launch<T, P, D>(a, ws, a.joined ? 0 : joins, splits, one, all, st);
}

// Whether some row tiles have a quarter more key tiles than they have on average.
template <int R, int KT, class A>
bool uneven(A& a) {
  int64_t keys, most = 0;
  const int64_t n = count_tiles<R, KT>(a, &keys);
  for (int i = 0; i < a.n_seqs; ++i) most = std::max(most, (int64_t)tiles_of<KT>(a.seq[i].nm) + tiles_of<KT>(tail_rows<R>(a, a.seq[i])));
  return 4 * most * n > 5 * keys;
}

// Many rows: units, and a join of the split row tiles.
template <typename T, typename P, int D, class A, typename One, typename All>
hipError_t launch_rounds(A& a, void* ws, int cus, double ends, double partial, One one, All all, hipStream_t st) {
  int64_t joins = plan_rounds<P::R, P::KT>(a, partials<P::R, D>(), cus, ends, partial);
  if (joins < 0) return hipErrorInvalidConfiguration;
  int splits = a.seq[0].splits;
  if constexpr (A::kPaged) {
    if (uneven<P::R, P::KT>(a)) {
      joins = plan_lengths<P::R, P::KT>(a, partials<P::R, D>(), cus, ends, partial);
      for (int i = 0; i < a.n_seqs; ++i) splits = std::max(splits, a.seq[i].splits);
    }
  }
  a.joined = 0;
  return launch<T, P, D>(a, ws, joins, splits, one, all, st);
}

template <int D, int NR, class A>
hipError_t attend_few_rows(A& a, int cus, void* ws, hipStream_t st) {
  if constexpr (A::kPaged) {
    bool memory = false;
    for (int i = 0; i < a.n_seqs; ++i) memory |= a.seq[i].nm > 0;
    if (!memory) {
      using P = Few<D, NR, 32>;
      return launch_shares<uint16_t, P, D>(a, ws, cus, attend_few<D, NR, typename A::One, 32>, attend_few<D, NR, A, 32>, st);
    }
  }
  using P = Few<D, NR>;
  return launch_shares<uint16_t, P, D>(a, ws, cus, attend_few<D, NR, typename A::One>, attend_few<D, NR, A>, st);
}

// A call whose largest sequence wants the many-row kernel has its sequences of
// up to `rows` query rows of a head (which never take it) taken out, for a
// launch of their own before it, if one of them has more keys than any other
// (its unit would end last) or they have more than 16 key tiles for each compute
// unit.  us, in one launch and in two, beside a chunk of 512 queries of 28 heads
// over 4608 keys: 7 tokens over 8292 keys 88 and 65, one over 1100 54 and 62;
// beside 2048 queries over 6144: 31 tokens over 16484 411 and 230, over 4196 (31
// tiles a CU) 214 and 189, 8 over 4196 (8) 164 and 176.
template <int R, int KT, class A>
A take_few(A& a, int rows, int cus) {
  A few = a, many = a;
  few.n_seqs = many.n_seqs = 0;
  int64_t longest[2] = {0, 0}, tiles;
  for (int i = 0; i < a.n_seqs; ++i) {
    const QuerySeq& s = a.seq[i];
    const bool is_few = (int64_t)a.group * s.nq <= rows;
    A& to = is_few ? few : many;
    to.seq[to.n_seqs++] = s;
    longest[is_few] = std::max(longest[is_few], (int64_t)s.nm + tail_rows<R>(a, s));
  }
  count_tiles<R, KT>(few, &tiles);
  if (longest[1] > longest[0] || tiles > 16 * cus) a = many; else few.n_seqs = 0;
  return few;
}

// Whether bf16 rows in pages take less time in units of 32 than in units of 256,
// where a head has 1024 at least (so that its keys are read by many units).  For
// the former: rounds of the chip (a single one, whose compute units have a unit
// each, hides less: 0.6 rounds more) times a unit's key tiles of 32, and the time
// of `ends` tiles for each round.  For the latter the longest unit's tiles of 64
// and 3 more, or the average and 11 with a join, or where there are more units than
// compute units the average and the last ones' difference; a window's borders are 2.  us,
// they and what they are taken for in brackets, width 128, 28 and 4 heads: a window
// of 100 over 1200 queries 29 (31) and 23 (19), over 500 14 (14) and 21 (19), of 1500
// over 300 37 (35) and 33 (33), prompts of 1000 34 (34) and 40 (40), of 2500 116 (112)
// and 88 (94), 400 queries over 2048 rows 44 (40) and 35 (37); width 64, 16 and 4
// heads: a prompt of 3000 56 (55) and 72 (66), windows of 100 over 2000 15 (15) and 17
// (16), over 4096 24 (26) and 18 (16), 400 queries over 8192 rows 64 (53) and 38 (39).
template <int D, class A>
bool fewer_rows_pay(const A& a, int cus) {
  constexpr double kFew = D == 128 ? 0.185 : 0.12, kMany = D == 128 ? 2.03 : 1.36;    // us of a tile
  constexpr double kEnds = D == 128 ? 24 : 20;
  double units = 0, keys = 0, blocks = 0, full = 0, half = 0, longest = 0;
  for (int i = 0; i < a.n_seqs; ++i) {
    const QuerySeq& s = a.seq[i];
    const double rows = (double)a.group * s.nq, n = a.h_kv * std::ceil(rows / 32), m = a.h_kv * std::ceil(rows / 256);
    const int near = tail_rows<32>(a, s);
    // (without a window a query sees half of its prompt on average; memory tiles of 128 take 2.6 tiles' time)
    const double seen = near < s.nt || s.v ? near : s.nq <= s.nt ? s.nt - s.nq / 2 : 0.5 * s.nt * s.nt / s.nq;
    const double held = std::ceil(s.nm / 64.0) + (near < s.nt ? 2 : 0), tiles = held + std::ceil(tail_rows<256>(a, s) / 64.0);
    units += n;
    keys += n * (std::ceil(seen / 32) + 2.6 * std::ceil(s.nm / 128.0));
    blocks += m;
    full += m * tiles;
    half += m * (held + std::min(tiles - held, std::ceil((seen + 64) / 64)));
    longest = std::max(longest, tiles);
  }
  const double rounds = std::ceil(units / cus), splits = std::max(1.0, std::floor(cus / units)), mean = keys / units / splits;
  const double few = (rounds + 0.6) * mean + kEnds * rounds + (splits > 1 ? 16 : 0);
  const double many = blocks < cus ? std::min(longest + 3, full / cus + 11) : (half + 3 * blocks) / cus + longest - half / blocks + 3;
  return kFew * few + 3 <= kMany * many + (D == 128 ? 3 : 5);
}

constexpr int kAlwaysFew = 64;   // query rows of a head that never take a many-row kernel
template <int D, class A>
hipError_t attend(const AttnDims& dm, A& a, int cus, void* ws, hipStream_t st) {
  int64_t rows = 0, memory = 0, tail = 0;
  for (int i = 0; i < a.n_seqs; ++i) {
    const QuerySeq& s = a.seq[i];
    const int64_t r = (int64_t)a.group * s.nq, tiles = a.h_kv * ((r + 31) / 32);
    rows = std::max(rows, r);
    memory += tiles * tiles_of<128>(s.nm);
    tail += tiles * tiles_of<128>(tail_rows<32>(a, s));
  }
  if (dm.dtype == OMNIMEM_F32) {
    // The few-row kernel up to 96 rows, to 192 over memories if the other's tiles of 128 would have a half more rows, and
    // where its tiles (32 rows and 128 keys) are at most 3 to a compute unit.  us, it and the many-row kernel, 4 heads,
    // 8 sequences of 32768 memory rows of width 64: 64 rows 232 and 329, 84 287 and 330, 112 450 and 330, 168 548 and 644;
    // of 8192 tail rows of width 128: 116 and 170, 181 and 171, 212 and 172, 328 and 314; one of 1500 tail rows of width
    // 64: 320 rows 17 and 23 (2 tiles), 500 19 and 22 (3), 1332 34 and 36 (8); of width 128: 25 and 28, 30 and 31, 65 and 57.
    // In pages at most 9 tiles for width 64: 1332 rows of 4 heads, a window of 250 16 and 24 (2), two sequences 27 and 33 (4),
    // four 42 and 46 (8), a window of 1000 31 and 34 (5), two 75 and 61 (10), without a window 37 and 39 (8), two 70 and 61
    // (16); width 128, 1600 rows of 2 heads, a window of 250 29 and 32 (2.3), 55 and 45 (4.7), of 1000 41 and 35 (3.1).
    if (rows <= 96 || (rows > 128 && rows <= 192 && memory >= tail) || memory + tail <= (A::kPaged && D == 64 ? 9 : 3) * cus)
      return launch_shares<float, F32<D>, D>(a, ws, cus, attend_f32<D, typename A::One>, attend_f32<D, A>, st);
    A few = take_few<F32Many<D>::R, F32Many<D>::KT>(a, kAlwaysFew, cus);
    if (few.n_seqs > 0) {
      const hipError_t e = attend<D>(dm, few, cus, ws, st);
      if (e != hipSuccess) return e;
    }
    return launch_rounds<float, F32Many<D>, D>(a, ws, cus, 1.0, 0.003, attend_f32_many<D, typename A::One>, attend_f32_many<D, A>, st);
  }
  if (rows <= 16) return attend_few_rows<D, 1>(a, cus, ws, st);
  if constexpr (A::kPaged) {
    // Units of 16 rows where a compute unit has one at most and 4 tail tiles (of 128 rows): half the instructions of those of
    // 32 one after the other.  us, 32 and 16 rows, 4 heads of width 128: trees of 28 rows of a head over 12 rows 7.9 and 6.2,
    // over 2000 11.2 and 9.8, of 112 rows over 500 10.8 and 9.6, four over up to 2000 16.0 and 15.5 (4), 448 rows over 500
    // 12.4 and 10.4 (2), over 2000 16.5 and 18.6 (7); 7 of 104 rows over 4096 memory rows of width 64 15.0 and 13.2, 16 of
    // them 19.1 and 17.2.
    int64_t units = 0, tiles = 0;
    for (int i = 0; i < a.n_seqs; ++i) {
      const int64_t n = a.h_kv * (((int64_t)a.group * a.seq[i].nq + 15) / 16);
      units += n;
      tiles += n * tiles_of<128>(tail_rows<16>(a, a.seq[i]));
    }
    if (units <= cus && tiles <= 4 * cus) return attend_few_rows<D, 1>(a, cus, ws, st);
  }
  // The few-row kernel up to 64 rows of a head, to 128 over memories (whose codes it reads again for each 32 rows at a
  // quarter of tail rows' cost), and where that leaves at most 40 tiles (32 rows and 128 memory rows, or 64 tail rows)
  // to a compute unit.  us, it and the many-row kernel, 4 heads of width 128: 56 rows, 8 sequences of 32768 memory rows
  // 61 and 120, of 8192 tail rows 37 and 50; 84 rows 83 and 122, 59 and 53 (48 tiles); 112 rows 105 and 125, 60 and 53
  // (64); 168 rows 137 and 130 (193), 74 and 55 (96); 448 rows over 8192 memory rows 24 and 34 (14), 8 sequences of 1024
  // tail rows 31 and 33 (28); 700 rows over 8192 33 and 35 (22), over 32768 73 and 65 (88).  In pages, whose lengths are
  // shared out evenly (plan_lengths), to 28: trees over 500 to 8192 rows, 448 rows of a head 32.0 and 32.0 (28; one
  // sequence), 42 and 38 (37; 2), 27.5 and 29.6 (14; 4 over up to 2048), 88 and 59 (98; 8), 224 rows 28 and 30 (18), 38 and
  // 35 (29); from 1024 rows on see fewer_rows_pay.
  bool is_few = rows <= kAlwaysFew || (rows <= 128 && memory >= tail) || memory + 2 * tail <= (A::kPaged ? 28 : 40) * cus;
  if constexpr (A::kPaged)
    if (rows >= 1024) is_few = fewer_rows_pay<D>(a, cus);
  if (is_few) return attend_few_rows<D, 2>(a, cus, ws, st);
  A few = take_few<Many<D>::R, Many<D>::KT>(a, kAlwaysFew, cus);
  if (few.n_seqs > 0) {
    const hipError_t e = attend<D>(dm, few, cus, ws, st);
    if (e != hipSuccess) return e;
  }
  return launch_rounds<uint16_t, Many<D>, D>(a, ws, cus, 3.0, 0.03, attend_many<D, typename A::One>, attend_many<D, A>, st);
}

template <typename Kernel>
hipError_t allow(Kernel kernel, int lds) {
  return lds <= 65536 ? hipSuccess : hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
}
// Lets the kernels for these arguments have the LDS that they need.
template <int D, class A>
hipError_t prepare() {
  hipError_t e = allow(attend_f32<D, A>, F32<D>::LDS);
  if (e == hipSuccess) e = allow(attend_f32_many<D, A>, F32Many<D>::LDS);
  if (e == hipSuccess) e = allow(attend_few<D, 1, A>, Few<D, 1>::LDS);
  if (e == hipSuccess) e = allow(attend_few<D, 2, A>, Few<D, 2>::LDS);
  if constexpr (A::kPaged) {
    if (e == hipSuccess) e = allow(attend_few<D, 1, A, 32>, Few<D, 1, 32>::LDS);
    if (e == hipSuccess) e = allow(attend_few<D, 2, A, 32>, Few<D, 2, 32>::LDS);
  }
  if (e == hipSuccess) e = allow(attend_many<D, A>, Many<D>::LDS);
  return e;
}
template <class A>
hipError_t prepare(const AttnDims& dm) {
  const hipError_t e = dm.d == 128 ? prepare<128, typename A::One>() : prepare<64, typename A::One>();
  return e != hipSuccess ? e : dm.d == 128 ? prepare<128, A>() : prepare<64, A>();
}
template <class A>
hipError_t attend_all(const AttnDims& dm, A& a, int n, int compute_units, void* ws, hipStream_t st) {
  a.n_seqs = n;
  a.h_kv = dm.h_kv;
  a.group = dm.group;
  return dm.d == 128 ? attend<128>(dm, a, compute_units, ws, st) : attend<64>(dm, a, compute_units, ws, st);
}

}  // namespace
}  // namespace omnimem
