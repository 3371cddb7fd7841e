// Internal declarations of the operators around the compression step
// (rotation, 4-bit memories, attention): descriptors as they travel to the
// kernels, and what the translation units share.
#pragma once

#include "common.h"

namespace omnimem {

// Sequences described by one launch: their descriptors are kernel arguments
// (of which a kernel may have 4 KiB), so a call needs no table on the device,
// no copy before it, and can be captured as it is.  The host writes arguments
// to device memory; a call for one sequence has a kernel with room for one
// (a token rotated, 3 KB and 0.9 KB of arguments: 8.9 and 8.2 us).
constexpr int kRotatesPerLaunch = 16, kHeldPerLaunch = 64, kQueriesPerLaunch = 32;

// ---------------------------------------------------------------------------
// 4-bit memories: blocks of 32 rows and 34 d bytes.
// ---------------------------------------------------------------------------
constexpr int kMemRows = 32;
template <int D>
struct MemBlock {
  static constexpr int BYTES = 34 * D;
  static constexpr int V = 16 * D, KS = 32 * D, VS = 33 * D;   // offsets: V codes, K scales, V scales
  static constexpr int PARTS = D / 32;                         // K groups of a row
  __host__ __device__ static inline int k_scale(int t, int p) { return KS + ((t & 3) * PARTS + p) * 8 + (t >> 2); }
  __host__ __device__ static inline int v_scale(int c) { return VS + (c & 15) * (D / 16) + (c >> 4); }
};
constexpr uint32_t kScaleNan = 255;    // the scale byte of a group with an infinity or NaN
constexpr uint32_t kScaleMin = 7, kScaleMax = 252;   // 2^-120 and 2^125
__device__ inline float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }

typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
__device__ inline uint2 gload8(const void* p) {
  const u32x2 v = gload<u32x2>(p);
  return make_uint2(v[0], v[1]);
}

// C consecutive elements of a row (4 or 8) as they lie in memory, and as fp32.
template <int C, typename T>
struct Raw {
  static constexpr int WORDS = C * (int)sizeof(T) / 4;
  uint32_t w[WORDS];
  __device__ inline void load(const T* p) {
#pragma unroll
    for (int i = 0; i < WORDS; i += 4) {
      if constexpr (WORDS == 2) {
        const uint2 y = gload8(p);
        w[0] = y.x; w[1] = y.y;
      } else {
        const uint4 y = gload16(reinterpret_cast<const uint32_t*>(p) + i);
        w[i] = y.x; w[i + 1] = y.y; w[i + 2] = y.z; w[i + 3] = y.w;
      }
    }
  }
  __device__ inline float operator[](int i) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
    return __uint_as_float(i & 1 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
  }
};

// The eight values (fp32) of a word of codes (the conversions give NaN where
// the scale is kScaleNan).
__device__ inline void values8(uint32_t w, uint32_t byte, float (&x)[8]) {
  const float s = scale_of(byte);
  const floatx2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 1);
  const floatx2 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 3);
  x[0] = a[0]; x[1] = a[1]; x[2] = b[0]; x[3] = b[1]; x[4] = c[0]; x[5] = c[1]; x[6] = d[0]; x[7] = d[1];
}
// The same as eight bf16 values (each is exact: three significant bits and an
// exponent of at least -121).
__device__ inline uint4 values8_bf16(uint32_t w, float scale) {
  uint4 r;
  r.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0));
  r.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1));
  r.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2));
  r.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3));
  return r;
}

// ---------------------------------------------------------------------------
// Kernel arguments.
// ---------------------------------------------------------------------------
struct RotateSeq {
  const void* q; const void* k; const void* v;
  const int32_t* pos;
  const uint8_t* mod;
  void* q_out; void* k_out; void* v_out;
  uint8_t* mod_out;
  int64_t q_hs, q_rs, kv_hs, kv_rs, pos_s, qo_hs, qo_rs, o_hs, o_rs;
  int64_t n;
};
template <int N>
struct RotateArgs {
  RotateSeq seq[N];
  double turns[64];            // inv_freq / 2 pi
  uint8_t axis[64];
  const void* q_w; const void* k_w;
  float eps;
  int rot, neighbours, h_q, h_kv;
};

struct HeldSeq {
  char* k; char* v; char* data;
  int64_t kv_hs, kv_rs, data_hs;
  int64_t n;
};
struct HeldArgs {
  HeldSeq seq[kHeldPerLaunch];
};

struct QuerySeq {
  const void* q; const char* mem; const void* k; const void* v;
  void* out; float* lse;
  uint32_t q_hs, q_rs, mem_hs, kv_hs, kv_rs, out_hs, out_rs;   // units of 16 bytes
  uint32_t lse_hs;             // elements
  float scale_log2;            // softmax scale times log2(e)
  int32_t nq, nm, nt;          // queries, memory rows, tail rows
  int32_t row_tiles, splits;   // of its work, see below
  int32_t slot0;               // its first partial (whole = 0)
};
// A call's work.  A KV head's query rows are numbered query-major (row
// i * G + h is query i of the head's h-th query head: neighbouring rows see
// the same keys, and share them), in tiles of R rows; row tiles are numbered
// over sequences, KV heads and rows.  A row tile's keys come in key tiles,
// the memory's and then the tail's.  A unit (one workgroup) takes a row tile
// and all its keys, or one of `splits` equal shares of them (few rows: of whole
// turns of its wavefronts, the last with what is left); then each writes
// a partial result (sums against its own maximum) and the join puts them
// together, in the order of the keys.  The first `whole` row tiles are not
// split (with whole > 0 all others are by the same number).
template <int N>
struct AttendArgs {
  static constexpr int kSeqs = N;
  static constexpr bool kPaged = false;
  using One = AttendArgs<1>;
  QuerySeq seq[N];
  int32_t unit0[N];            // a sequence's first unit after the whole row tiles (whole = 0), or row tile
  int n_seqs, h_kv, group, causal, whole, units;
  int joined;                  // the last unit of a row tile joins its partials
  float* part_o;               // [partials][R][d] unnormalised sums
  float2* part_ml;             // [partials][R] (maximum in log2 units, sum of weights)
  int* arrived;                // [partials] units of the row tile (at its first partial) that wrote theirs; 0 between calls
};
static_assert(sizeof(RotateArgs<kRotatesPerLaunch>) <= 3968 && sizeof(HeldArgs) <= 3968 && sizeof(AttendArgs<kQueriesPerLaunch>) <= 3968,
              "a kernel's arguments, with what the runtime adds, stay below 4 KiB");

// A cache in pages, in bytes.  Row r of a sequence is row r % (1 << shift) of
// page table[r >> shift]; an entry that is not below n_pages is no page.
struct PagePool {
  char* k; char* v;
  int64_t page, head;          // from a page (a head) to the next
  uint32_t row;                // below 2^24
  uint32_t n_pages;
  int shift;                   // 4 to 8: 16 rows from a multiple of 16 lie on one page
};
// Byte of a head's row of the cache from that head's first row on page 0, below
// 0 if it has no page (a store spans less than 64 TiB).  SAME: of one row in
// every lane, whose entry is a scalar load.
template <bool SAME>
__device__ inline int64_t paged_row(const PagePool& pool, const int32_t* table, int row) {
  uint32_t entry;
  if constexpr (SAME) entry = ((const __attribute__((address_space(4))) uint32_t*)(uintptr_t)table)[uniform(row) >> pool.shift];
  else entry = gload<uint32_t>(table + (row >> pool.shift));
  return entry < pool.n_pages ? entry * pool.page + (row & ((1 << pool.shift) - 1)) * (int64_t)pool.row : INT64_MIN;
}
struct PagedRotateSeq {
  const void* q; const void* k; const void* v;
  const int32_t* pos;
  void* q_out;
  const int32_t* table;
  int64_t pos_s;
  uint32_t q_hs, q_rs, kv_hs, kv_rs, qo_hs, qo_rs;   // units of 16 bytes
  int32_t first, n;
};
template <int N>
struct PagedRotateArgs {
  PagedRotateSeq seq[N];
  PagePool pool;
  double turns[64];
  uint8_t axis[64];
  const void* q_w; const void* k_w;
  float eps;
  int rot, neighbours, h_q, h_kv, n_axes;
  int waves;                   // to a token
};
constexpr int kPagedRotatesPerLaunch = 32;

// Accepted drafts: `skip` rows are in their place, the others move.
constexpr int kKeptPerLaunch = 36, kStoresPerLaunch = 32, kMaxDrafts = 64;
struct KeptSeq {
  const int32_t* table;
  int32_t first;
  uint8_t skip, n;
  uint8_t path[kMaxDrafts];
};
struct KeepArgs {
  KeptSeq seq[kKeptPerLaunch];
  char* k[kStoresPerLaunch];
  char* v[kStoresPerLaunch];
  PagePool pool;               // (k, v: not used)
};
static_assert(sizeof(PagedRotateArgs<kPagedRotatesPerLaunch>) <= 3968 && sizeof(KeepArgs) <= 3968, "as above");

// Attention's arguments for tail rows in pages: a sequence's `k` is its table and its `v`
// its drafts' masks, or null.
template <int N>
struct PagedArgs : AttendArgs<N> {
  static constexpr bool kPaged = true;
  using One = PagedArgs<1>;
  PagePool pool;
  int32_t window, sinks;       // at most 2^30
};
static_assert(sizeof(PagedArgs<kQueriesPerLaunch>) <= 3968, "as above");

struct AttnDims {
  int h_q, h_kv, group, d, dtype;
};
// (a: room for the most; the launch takes what n sequences need)
hipError_t launch_rotate(const AttnDims& dm, const RotateArgs<kRotatesPerLaunch>& a, int n, hipStream_t st);
hipError_t launch_rotate_pages(const AttnDims& dm, const PagedRotateArgs<kPagedRotatesPerLaunch>& a, int n, hipStream_t st);
hipError_t launch_keep(const AttnDims& dm, const KeepArgs& a, int n, int stores, hipStream_t st);
hipError_t launch_hold(const AttnDims& dm, const HeldArgs& a, int n, bool pack, hipStream_t st);
// Workspace of a handle: partials, then a counter for each (all 0 at first).
constexpr int64_t kPartBytes = (int64_t)128 << 20, kMaxPartials = 32768;
// Lets the kernels of these sizes have the LDS that they need, on the current device.
hipError_t prepare_attend(const AttnDims& dm);
// Fills the plan fields of `a` for n sequences and launches their attention.
hipError_t launch_attend(const AttnDims& dm, AttendArgs<kQueriesPerLaunch>& a, int n, int compute_units, void* workspace, hipStream_t st);
hipError_t prepare_attend_pages(const AttnDims& dm);
hipError_t launch_attend_pages(const AttnDims& dm, PagedArgs<kQueriesPerLaunch>& a, int n, int compute_units, void* workspace, hipStream_t st);

}  // namespace omnimem
