// A chunk's projected rows to the pages of a cache: per-head norm and rotation
// of queries and keys, values copied, in one pass.
#include <cstddef>
#include <cstring>

#include "../../include/omnimem.h"
#include "rotate.h"

namespace omnimem {
namespace {

template <typename T>
__device__ inline int64_t elems(uint32_t units) { return (int64_t)units * (16 / (int)sizeof(T)); }
// Channels of a lane's run: 16 bytes, so that neighbouring lanes write next to
// each other.
template <typename T>
constexpr int kRun = 16 / (int)sizeof(T);

// Few tokens: a workgroup to a token, its heads side by side in the lanes of as
// many wavefronts as they fill.  What a lane waits for, its rows, the table's
// entry, the token's positions, its frequency and that one's axis, depends on
// the arguments alone and is asked for at once; the cosines are formed while the
// rows are on their way.  Latency bounds it: 32 tokens of 36 heads of width 128
// take 4.0 us a launch on the device, of which an empty one has 3.1 (without the
// stores 3.7); 2331 of 20 heads of width 64 in fp32 (23.9 MB) 9.4, where loads,
// 3.2, and stores, 4.4, follow one another in all wavefronts at once (with runs
// of 32 bytes to a lane 12.1).
constexpr int kRowWaves = 12;    // at most
template <typename T, int D, class A>
__global__ __launch_bounds__(64 * kRowWaves) void rotate_row(A a) {
  constexpr int C = kRun<T>, U = D / (2 * C), HEADS = 64 / U;
  const PagedRotateSeq& s = a.seq[blockIdx.y];
  const int lane = threadIdx.x & 63, wave = wave_id(), step = a.waves * HEADS;
  const int t = blockIdx.x;
  if (t >= s.n) return;
  const int h_q = a.h_q, h_kv = a.h_kv, heads = h_q + 2 * h_kv;
  const Part<T, D, C> shape(lane % U, a.rot, a.neighbours);
  const T* src;
  char* dst;
  const T* w;
  Raw<C, T> x = {}, y = {}, wx = {}, wy = {};
  const int64_t to = paged_row<true>(a.pool, s.table, s.first + t);
  const auto load = [&](int h) __attribute__((always_inline)) {
    const int kind = h < h_q ? 0 : h < h_q + h_kv ? 1 : 2, g = kind == 0 ? h : kind == 1 ? h - h_q : h - h_q - h_kv;
    src = static_cast<const T*>(kind == 0 ? s.q : kind == 1 ? s.k : s.v) +
          (kind == 0 ? g * elems<T>(s.q_hs) + t * elems<T>(s.q_rs) : g * elems<T>(s.kv_hs) + t * elems<T>(s.kv_rs));
    w = static_cast<const T*>(kind == 0 ? a.q_w : kind == 1 ? a.k_w : nullptr);
    x.load(src + shape.ca);
    y.load(src + shape.cb);
    if (w) {
      wx.load(w + shape.ca);
      wy.load(w + shape.cb);
    }
    dst = kind == 0 ? static_cast<char*>(s.q_out) + (g * elems<T>(s.qo_hs) + t * elems<T>(s.qo_rs)) * (int)sizeof(T)
                    : (kind == 1 ? a.pool.k : a.pool.v) + g * a.pool.head + to;
  };
  int h = wave * HEADS + lane / U;
  if (h < heads) load(h);
  typedef const __attribute__((address_space(4))) int32_t scalar_t;
  const scalar_t* pos = (scalar_t*)(uintptr_t)s.pos;
  int p[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) p[i] = pos[min(i, a.n_axes - 1) * s.pos_s + t];
  const int axis = a.axis[lane];
  const double turns = a.turns[lane];
  asm volatile("" ::: "memory");           // (all of it is on its way before the first is waited for)
  floatx2 mine = floatx2{1.0f, 0.0f};
  if (lane < a.rot / 2) mine = turn_of(axis == 0 ? p[0] : axis == 1 ? p[1] : axis == 2 ? p[2] : p[3], turns);
  Part<T, D, C> part = shape;
#pragma unroll
  for (int i = 0; i < C; ++i) {
    part.c[i] = __shfl(mine[0], lane % U * C + i);
    part.s[i] = __shfl(mine[1], lane % U * C + i);
  }
  while (h < heads) {
    part.finish(x, y, w != nullptr, wx, wy, a.eps, h < h_q + h_kv, reinterpret_cast<T*>(dst), h < h_q || to >= 0);
    h += step;
    if (h < heads) load(h);
  }
}

// Many tokens: a workgroup to as many neighbouring tokens as a wavefront has rows, a head of all of
// them to a wavefront at a time, as rotate_tokens.  Bandwidth bounds it: 16384
// tokens of 36 heads of width 128 (302 MB read and written) take 63 us, 4.8 TB/s.
template <typename T, int D, class A>
__global__ __launch_bounds__(256) void rotate_rows(A a) {
  constexpr int C = kRun<T>, U = D / (2 * C), TOKENS = 64 / U, F = D / 2;
  const PagedRotateSeq& s = a.seq[blockIdx.y];
  const int lane = threadIdx.x & 63, wave = wave_id();
  const int t0 = blockIdx.x * TOKENS;
  if (t0 >= s.n) return;
  __shared__ floatx2 turn[TOKENS][F];
  for (int e = threadIdx.x; e < TOKENS * F; e += 256) {
    const int i = e / F, j = e % F;
    if (j < a.rot / 2 && t0 + i < s.n) turn[i][j] = turn_of(gload<int32_t>(s.pos + a.axis[j] * s.pos_s + t0 + i), a.turns[j]);
  }
  __syncthreads();
  const int tok = lane / U, u = lane % U;
  const bool live = t0 + tok < s.n;
  const int t = min(t0 + tok, s.n - 1);
  Part<T, D, C> part(u, a.rot, a.neighbours);
#pragma unroll
  for (int i = 0; i < C; ++i) {
    const floatx2 y = part.turns && live ? turn[tok][u * C + i] : floatx2{1.0f, 0.0f};
    part.c[i] = y[0];
    part.s[i] = y[1];
  }
  const int h_q = a.h_q, h_kv = a.h_kv, heads = h_q + 2 * h_kv;
  const T* q_w = static_cast<const T*>(a.q_w);
  const T* k_w = static_cast<const T*>(a.k_w);
  Raw<C, T> qx = {}, qy = {}, kx = {}, ky = {}, x, y;
  if (q_w) { qx.load(q_w + part.ca); qy.load(q_w + part.cb); }
  if (k_w) { kx.load(k_w + part.ca); ky.load(k_w + part.cb); }
  const int64_t tq = t * elems<T>(s.q_rs), tkv = t * elems<T>(s.kv_rs), tqo = t * elems<T>(s.qo_rs);
  const int64_t q_hs = elems<T>(s.q_hs), kv_hs = elems<T>(s.kv_hs), to = paged_row<false>(a.pool, s.table, s.first + t);
  const auto load = [&](int h) __attribute__((always_inline)) {
    const T* p = h < h_q ? static_cast<const T*>(s.q) + h * q_hs + tq
                         : static_cast<const T*>(h < h_q + h_kv ? s.k : s.v) + (h - h_q - (h < h_q + h_kv ? 0 : h_kv)) * kv_hs + tkv;
    x.load(p + part.ca);
    y.load(p + part.cb);
  };
  int h = wave;
  if (h < heads) load(h);
  for (; h < heads; h += 4) {
    const Raw<C, T> cx = x, cy = y;
    if (h + 4 < heads) load(h + 4);
    if (h < h_q)
      part.finish(cx, cy, q_w != nullptr, qx, qy, a.eps, true, static_cast<T*>(s.q_out) + h * elems<T>(s.qo_hs) + tqo, live);
    else if (h < h_q + h_kv)
      part.finish(cx, cy, k_w != nullptr, kx, ky, a.eps, true, reinterpret_cast<T*>(a.pool.k + (h - h_q) * a.pool.head + to), live && to >= 0);
    else
      part.finish(cx, cy, false, kx, ky, a.eps, false, reinterpret_cast<T*>(a.pool.v + (h - h_q - h_kv) * a.pool.head + to), live && to >= 0);
  }
}

using All = PagedRotateArgs<kPagedRotatesPerLaunch>;
template <typename T, int D, int N>
void launch(const All& a, int n, int64_t rows, int64_t tokens, hipStream_t st) {
  PagedRotateArgs<N> x;
  std::memcpy(x.seq, a.seq, N * sizeof a.seq[0]);
  x.pool = a.pool;
  std::memcpy(x.turns, a.turns, sizeof a - offsetof(All, turns));
  constexpr int U = D / (2 * kRun<T>), TOKENS = 64 / U;
  // us, a workgroup to a token and to several: 2000 tokens of 36 heads of width 128 11.4 and 13.1, 4000 17.4 and 16.1; of 12
  // heads 6.6 and 7.2, 11.1 and 9.2; of 24 heads of width 64 6.5 and 9.1, 10.9 and 10.4; 20 heads of fp32, width 64: 1000 5.2
  // and 6.9, 2331 9.2 and 8.9, 3500 11.1 and 9.9.  The grid is the longest sequence times the sequences: prompts of 1000, 2900
  // and 4000 (36 heads of width 128, in a graph on one state) 5.7, 12.7 and 14.4, beside 31 tokens of other sequences 11.4, 30.0
  // and 20.2
  if (tokens >= 3000) {
    rotate_rows<T, D, PagedRotateArgs<N>><<<dim3((unsigned)((rows + TOKENS - 1) / TOKENS), n), 256, 0, st>>>(x);
  } else {
    // wavefronts for all heads of a token, as long as the chip has them side by side; us, 36 heads of width 128, 5 and 4 or 2:
    // 256 tokens 4.8 and 5.6, 1000 9.0 and 8.1 (2: 8.7), 2000 14.6 and 11.4 (4: 12.7)
    const int all = (a.h_q + 2 * a.h_kv + TOKENS - 1) / TOKENS;
    const int waves = std::min({all, kRowWaves, std::max(2, (int)(4096 / tokens))});
    x.waves = waves;
    rotate_row<T, D, PagedRotateArgs<N>><<<dim3((unsigned)rows, n), 64 * waves, 0, st>>>(x);
  }
}
// (arguments are written to device memory by the host: room for 1, 8 or all sequences)
template <typename T, int D>
void launch(const All& a, int n, int64_t rows, int64_t tokens, hipStream_t st) {
  if (n == 1) launch<T, D, 1>(a, n, rows, tokens, st);
  else if (n <= 8) launch<T, D, 8>(a, n, rows, tokens, st);
  else launch<T, D, kPagedRotatesPerLaunch>(a, n, rows, tokens, st);
}

}  // namespace

hipError_t launch_rotate_pages(const AttnDims& dm, const All& a, int n, hipStream_t st) {
  int64_t rows = 0, tokens = 0;
  for (int i = 0; i < n; ++i) {
    rows = std::max<int64_t>(rows, a.seq[i].n);
    tokens += a.seq[i].n;
  }
  if (rows == 0) return hipSuccess;
  if (dm.dtype == OMNIMEM_BF16) {
    if (dm.d == 128) launch<uint16_t, 128>(a, n, rows, tokens, st); else launch<uint16_t, 64>(a, n, rows, tokens, st);
  } else {
    if (dm.d == 128) launch<float, 128>(a, n, rows, tokens, st); else launch<float, 64>(a, n, rows, tokens, st);
  }
  return hipGetLastError();
}

}  // namespace omnimem
