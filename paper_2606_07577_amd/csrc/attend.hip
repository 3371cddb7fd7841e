// Attention over a 4-bit memory and the tail rows behind it.
#include "../../include/omnimem.h"
#include "attn.h"

namespace omnimem {
namespace {

// Where a unit's work lies.
struct Unit {
  int s, g, rt, split;       // sequence, KV head, row tile, split
  int rows;                  // query rows of the head (G * n_q)
  int k0, k1;                // key tiles
  int mem_tiles;             // of the sequence
  int slot;                  // partial, or -1: the result is final
};

// Tail rows that query i sees.
__device__ inline int tail_seen(const QuerySeq& s, int causal, int i) {
  return causal ? min(max(s.nt - s.nq + i + 1, 0), s.nt) : s.nt;
}
__host__ __device__ inline int tiles_of(int64_t rows) { return (int)((rows + kKeyTile - 1) / kKeyTile); }

template <int R>
__device__ inline Unit unit_of(const AttendArgs& a, int u) {
  Unit x;
  x.s = 0;
  while (x.s + 1 < a.n_seqs && u >= a.seq[x.s + 1].unit0) ++x.s;
  const QuerySeq& s = a.seq[x.s];
  u -= s.unit0;
  x.slot = s.splits > 1 ? s.slot0 + u : -1;
  x.split = u % s.splits;
  u /= s.splits;
  x.rt = u % s.row_tiles;
  x.g = u / s.row_tiles;
  x.rows = a.group * s.nq;
  x.mem_tiles = tiles_of(s.nm);
  const int last = (min((x.rt + 1) * R, x.rows) - 1) / a.group;   // the tile's last query sees the most
  const int tiles = x.mem_tiles + tiles_of(tail_seen(s, a.causal, last));
  x.k0 = min(x.split * a.chunk, tiles);
  x.k1 = min(x.k0 + a.chunk, tiles);
  return x;
}

template <typename T> __device__ inline float to_f32(T x);
template <> __device__ inline float to_f32(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
template <> __device__ inline float to_f32(float x) { return x; }
__device__ inline void put(uint16_t* p, float x) { *p = (uint16_t)round2(x, 0.0f); }
__device__ inline void put(float* p, float x) { *p = x; }
template <typename T> __device__ inline T as(float x);
template <> __device__ inline uint16_t as<uint16_t>(float x) { return (uint16_t)round2(x, 0.0f); }
template <> __device__ inline float as<float>(float x) { return x; }

__device__ inline float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

// The simple form: 32 query rows to a unit; the four wavefronts take 32 keys
// each of a tile of 128 in LDS, and join their sums at the end.
template <typename T, int D>
struct Simple {
  static constexpr int R = 32;
  static constexpr int ROW = D + 16 / (int)sizeof(T);      // padded LDS row
  static constexpr int LDS = 2 * kKeyTile * ROW * (int)sizeof(T) + 4 * R * 8;
};

template <typename T, int D>
__global__ __launch_bounds__(256) void attend_simple(AttendArgs a) {
  using P = Simple<T, D>;
  using M = Mfma<T>;
  using frag = typename M::frag;
  constexpr int R = P::R, ROW = P::ROW, NKS = D / M::KSTEP, NCT = D / 32;
  using B = MemBlock<D>;
  extern __shared__ __align__(16) char lds[];
  T* kt = reinterpret_cast<T*>(lds);
  T* vt = kt + kKeyTile * ROW;
  float2* ml = reinterpret_cast<float2*>(lds + 2 * kKeyTile * ROW * sizeof(T));   // [4][R]
  const Unit x = unit_of<R>(a, blockIdx.x);
  const QuerySeq& s = a.seq[x.s];
  const int lane = threadIdx.x & 63, wave = wave_id(), half = lane >> 5, col = lane & 31;
  const int row = x.rt * R + col;
  const bool live = row < x.rows;
  const int i = live ? row / a.group : 0, hh = row - i * a.group;
  const int h = x.g * a.group + (live ? hh : 0);
  const int seen = live ? tail_seen(s, a.causal, i) : 0;
  const T* q = static_cast<const T*>(s.q) + h * s.q_hs + i * s.q_rs;
  frag qf[NKS];
#pragma unroll
  for (int ks = 0; ks < NKS; ++ks) qf[ks] = live ? M::gload(q + ks * M::KSTEP + half * M::PER_LANE) : M::zero();

  floatx16 o[NCT];
#pragma unroll
  for (int c = 0; c < NCT; ++c) o[c] = floatx16{};
  float m = -INFINITY, l = 0.0f;

  for (int kti = x.k0; kti < x.k1; ++kti) {
    __syncthreads();
    const bool in_mem = kti < x.mem_tiles;
    const int key0 = (in_mem ? kti : kti - x.mem_tiles) * kKeyTile;
    const int keys = min(kKeyTile, (in_mem ? s.nm : s.nt) - key0);
    if (in_mem) {
      const char* data = s.mem + x.g * s.mem_hs + (int64_t)(key0 / kMemRows) * B::BYTES;
      const int blocks = (keys + kMemRows - 1) / kMemRows;
      for (int e = threadIdx.x; e < kKeyTile * D / 8; e += 256) {
        const int t = e / (D / 8), c8 = e % (D / 8), b = t / kMemRows;
        float y[8] = {};
        if (b < blocks) {
          const char* blk = data + (int64_t)b * B::BYTES;
          values8(gload<uint32_t>(blk + (t % kMemRows) * (D / 2) + c8 * 4), gload<uint8_t>(blk + B::k_scale(t % kMemRows, c8 >> 2)), y);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) kt[t * ROW + c8 * 8 + j] = as<T>(y[j]);
      }
      for (int e = threadIdx.x; e < kKeyTile * D / 8; e += 256) {
        const int c = e % D, t8 = e / D, b = t8 / 4;
        float y[8] = {};
        if (b < blocks) {
          const char* blk = data + (int64_t)b * B::BYTES;
          values8(gload<uint32_t>(blk + B::V + c * 16 + (t8 & 3) * 4), gload<uint8_t>(blk + B::v_scale(c)), y);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) vt[(t8 * 8 + j) * ROW + c] = as<T>(y[j]);
      }
    } else {
      constexpr int E = 16 / (int)sizeof(T);
      const T* k = static_cast<const T*>(s.k) + x.g * s.kv_hs + key0 * s.kv_rs;
      const T* v = static_cast<const T*>(s.v) + x.g * s.kv_hs + key0 * s.kv_rs;
      for (int e = threadIdx.x; e < kKeyTile * D / E; e += 256) {
        const int t = e / (D / E), c = e % (D / E) * E;
        const uint4 z = make_uint4(0, 0, 0, 0);
        *reinterpret_cast<uint4*>(kt + t * ROW + c) = t < keys ? gload16(k + t * s.kv_rs + c) : z;
        *reinterpret_cast<uint4*>(vt + t * ROW + c) = t < keys ? gload16(v + t * s.kv_rs + c) : z;
      }
    }
    __syncthreads();
    floatx16 sc = floatx16{};
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks) {
      const T* kp = kt + (wave * 32 + col) * ROW + ks * M::KSTEP + half * M::PER_LANE;
      sc = M::mma(M::load(kp), qf[ks], sc);
    }
    const int limit = in_mem ? (live ? keys : 0) : seen - key0;
    float top = -INFINITY;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int key = wave * 32 + acc_row(r, lane);
      sc[r] = key < limit ? sc[r] * s.scale_log2 : -INFINITY;
      top = fmaxf(top, sc[r]);
    }
    top = fmaxf(top, __shfl_xor(top, 32));
    const float m2 = fmaxf(m, top), ref = m2 == -INFINITY ? 0.0f : m2;
    const float alpha = exp2_(m - ref);
    m = m2;
    float sum = 0.0f;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      sc[r] = exp2_(sc[r] - ref);
      sum += sc[r];
    }
    l = l * alpha + sum;
#pragma unroll
    for (int c = 0; c < NCT; ++c) o[c] *= alpha;
    // keys of accumulator registers r .. of this half: (r >> 2) * 8 + half * 4 + (r & 3)
#pragma unroll
    for (int c = 0; c < NCT; ++c) {
      const T* vp = vt + (wave * 32 + half * 4) * ROW + c * 32 + col;
      if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
          uint32_t va[4], pa[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int t = kk * 16 + (j >> 1) * 8 + (j & 1) * 2;
            va[j] = (uint32_t)vp[t * ROW] | ((uint32_t)vp[(t + 1) * ROW] << 16);
            pa[j] = round2(sc[kk * 8 + 2 * j], sc[kk * 8 + 2 * j + 1]);
          }
          o[c] = M::mma(__builtin_bit_cast(frag, make_uint4(va[0], va[1], va[2], va[3])),
                        __builtin_bit_cast(frag, make_uint4(pa[0], pa[1], pa[2], pa[3])), o[c]);
        }
      } else {
#pragma unroll
        for (int r = 0; r < 16; ++r) o[c] = M::mma(vp[((r >> 2) * 8 + (r & 3)) * ROW], sc[r], o[c]);
      }
    }
  }
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
  float* ob = reinterpret_cast<float*>(lds);       // [R][D + 4], the tiles are done with
  constexpr int OROW = D + 4;
  for (int w = 0; w < 4; ++w) {
    __syncthreads();
    if (wave == w) {
#pragma unroll
      for (int c = 0; c < NCT; ++c)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          float* p = ob + col * OROW + c * 32 + acc_row(r, lane);
          const float y = o[c][r] * mine;
          *p = w == 0 ? y : *p + y;
        }
    }
  }
  __syncthreads();
  if (x.slot >= 0) {
    float* po = a.part_o + (int64_t)x.slot * R * D;
    for (int e = threadIdx.x; e < R * D; e += 256) po[e] = ob[e / D * OROW + e % D];
    if (threadIdx.x < R) a.part_ml[(int64_t)x.slot * R + threadIdx.x] = make_float2(top, total);
  } else {
    float* inv = reinterpret_cast<float*>(ml);
    __syncthreads();
    if (threadIdx.x < R) {
      inv[threadIdx.x] = total == 0.0f ? 0.0f : 1.0f / total;
      if (live && s.lse) s.lse[h * s.lse_hs + i] = total == 0.0f ? -INFINITY : (top + log2f(total)) * kLn2;
    }
    __syncthreads();
    for (int e = threadIdx.x; e < R * D; e += 256) {
      const int r = e / D, c = e % D, gr = x.rt * R + r;
      if (gr >= x.rows) break;
      const int qi = gr / a.group, qh = x.g * a.group + gr % a.group;
      put(static_cast<T*>(s.out) + qh * s.out_hs + qi * s.out_rs + c, ob[r * OROW + c] * inv[r]);
    }
  }
}

// Puts the partial results of a query row's splits together: a workgroup per
// row, D/4 threads to a partial.
template <typename T, int D, int R>
__global__ __launch_bounds__(256) void join_splits(AttendArgs a) {
  constexpr int TPR = D / 4, PAR = 256 / TPR;
  __shared__ floatx4 sums[PAR][TPR];
  __shared__ float2 stat[4];
  int u = blockIdx.x, si = 0;
  for (; si + 1 < a.n_seqs; ++si) {
    const int n = a.seq[si].splits > 1 ? a.h_kv * a.seq[si].row_tiles : 0;
    if (u < n) break;
    u -= n;
  }
  const QuerySeq& s = a.seq[si];
  const int rt = u % s.row_tiles, g = u / s.row_tiles;
  const int row = rt * R + blockIdx.y;
  if (row >= a.group * s.nq) return;
  const int i = row / a.group, h = g * a.group + row % a.group;
  const int64_t slot = s.slot0 + (int64_t)u * s.splits;
  const float2* ml = a.part_ml + slot * R + blockIdx.y;
  float m = -INFINITY;
  for (int p = threadIdx.x; p < s.splits; p += 256) m = fmaxf(m, gload<float>(&ml[(int64_t)p * R].x));
#pragma unroll
  for (int k = 1; k < 64; k *= 2) m = fmaxf(m, __shfl_xor(m, k));
  if ((threadIdx.x & 63) == 0) stat[threadIdx.x >> 6].x = m;
  __syncthreads();
  m = fmaxf(fmaxf(stat[0].x, stat[1].x), fmaxf(stat[2].x, stat[3].x));
  const float ref = m == -INFINITY ? 0.0f : m;
  const int c = threadIdx.x % TPR, p0 = threadIdx.x / TPR;
  floatx4 o = floatx4{};
  float l = 0.0f;
  for (int p = p0; p < s.splits; p += PAR) {
    const floatx2 x = gload<floatx2>(&ml[(int64_t)p * R]);
    if (x[0] == -INFINITY) continue;           // (it may have written no sums)
    const float w = exp2_(x[0] - ref);
    l += w * x[1];
    o += w * gload<floatx4>(a.part_o + ((slot + p) * R + blockIdx.y) * D + c * 4);
  }
  sums[p0][c] = o;
  __shared__ float ls[PAR];
  if (c == 0) ls[p0] = l;
  __syncthreads();
  if (threadIdx.x >= TPR) return;
  l = 0.0f;
  o = floatx4{};
#pragma unroll
  for (int p = 0; p < PAR; ++p) { o += sums[p][c]; l += ls[p]; }
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  T* out = static_cast<T*>(s.out) + h * s.out_hs + i * s.out_rs + c * 4;
  if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2*>(out) = make_uint2(round2(o[0] * inv, o[1] * inv), round2(o[2] * inv, o[3] * inv));
  else *reinterpret_cast<floatx4*>(out) = o * inv;
  if (c == 0 && s.lse) s.lse[h * s.lse_hs + i] = l == 0.0f ? -INFINITY : (m + log2f(l)) * kLn2;
}

// Row tiles of R rows, key tiles in chunks: as few units as fill the chip
// (`target`), no more partials than the workspace holds.
template <int R, int D>
int plan(AttendArgs& a, int n, int h_kv, int64_t target) {
  int64_t most = 1, tiles_all = 0;
  for (int i = 0; i < n; ++i) {
    QuerySeq& s = a.seq[i];
    s.row_tiles = (int)(((int64_t)a.group * s.nq + R - 1) / R);
    const int64_t t = std::max(tiles_of(s.nm) + tiles_of(s.nt), 1);
    most = std::max(most, t);
    tiles_all += (int64_t)h_kv * s.row_tiles * t;
  }
  const int64_t slots = kPartBytes / (R * (D * 4 + 8));
  int64_t chunk = std::max<int64_t>(1, tiles_all / target);
  for (;; chunk += 1 + chunk / 16) {
    int64_t units = 0, parts = 0;
    for (int i = 0; i < n; ++i) {
      QuerySeq& s = a.seq[i];
      const int64_t t = std::max(tiles_of(s.nm) + tiles_of(s.nt), 1);
      s.splits = (int)((t + chunk - 1) / chunk);
      s.unit0 = (int)units;
      s.slot0 = (int)parts;
      const int64_t u = (int64_t)h_kv * s.row_tiles * s.splits;
      units += u;
      if (s.splits > 1) parts += u;
      if (units > INT32_MAX) return -1;
    }
    if (parts <= slots) {
      a.chunk = (int)chunk;
      return (int)units;
    }
  }
}

template <typename T, int D>
hipError_t attend(AttendArgs& a, int n, int compute_units, void* ws, hipStream_t st) {
  using P = Simple<T, D>;
  constexpr int R = P::R;
  const int units = plan<R, D>(a, n, a.h_kv, 4 * compute_units);
  a.part_o = static_cast<float*>(ws);
  a.part_ml = reinterpret_cast<float2*>(a.part_o + (int64_t)(kPartBytes / (R * (D * 4 + 8))) * R * D);
  if (units < 0) return hipErrorInvalidConfiguration;
  hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(attend_simple<T, D>), hipFuncAttributeMaxDynamicSharedMemorySize, P::LDS);
  if (e != hipSuccess) return e;
  attend_simple<T, D><<<units, 256, P::LDS, st>>>(a);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  int joins = 0;
  for (int i = 0; i < n; ++i)
    if (a.seq[i].splits > 1) joins += a.h_kv * a.seq[i].row_tiles;
  if (joins) join_splits<T, D, R><<<dim3(joins, R), 256, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_attend(const AttnDims& dm, AttendArgs& a, int n, int compute_units, void* ws, hipStream_t st) {
  a.n_seqs = n;
  a.h_kv = dm.h_kv;
  a.group = dm.group;
  if (dm.dtype == OMNIMEM_BF16)
    return dm.d == 128 ? attend<uint16_t, 128>(a, n, compute_units, ws, st) : attend<uint16_t, 64>(a, n, compute_units, ws, st);
  return dm.d == 128 ? attend<float, 128>(a, n, compute_units, ws, st) : attend<float, 64>(a, n, compute_units, ws, st);
}

}  // namespace omnimem
