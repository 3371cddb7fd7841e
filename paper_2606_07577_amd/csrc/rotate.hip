// A chunk's projected rows to their places behind the cache: per-head norm
// and rotation of queries and keys, values copied, in one pass.
#include <cstddef>
#include <cstring>

#include "../../include/omnimem.h"
#include "attn.h"

namespace omnimem {
namespace {

__device__ inline void store8(uint16_t* p, const float (&x)[8]) {
  *reinterpret_cast<uint4*>(p) = make_uint4(round2(x[0], x[1]), round2(x[2], x[3]), round2(x[4], x[5]), round2(x[6], x[7]));
}
__device__ inline void store8(float* p, const float (&x)[8]) {
  *reinterpret_cast<floatx4*>(p) = floatx4{x[0], x[1], x[2], x[3]};
  *reinterpret_cast<floatx4*>(p + 4) = floatx4{x[4], x[5], x[6], x[7]};
}

// Cosine and sine of a position times a frequency in turns, formed and reduced
// in 64 bits.
__device__ inline floatx2 turn_of(int32_t pos, double turns) {
  const double x = (double)pos * turns;
  float c, s;
  sincospif(2.0f * (float)(x - rint(x)), &s, &c);
  return floatx2{c, s};
}

// A lane's 16 channels of a row: two runs of 8 that turn with 8 frequencies
// (against each other, or neighbours within them), D/16 lanes to a row.
template <typename T, int D>
struct Part {
  static constexpr int U = D / 16;
  int ca, cb;                // first channels of the runs
  bool turns, half;
  float c[8], s[8];
  __device__ inline Part(int u, int rot, int neighbours) {
    turns = u < rot / 16;
    half = turns && !neighbours;
    ca = half ? 8 * u : 16 * u;
    cb = half ? rot / 2 + 8 * u : 16 * u + 8;
  }
  // Normalises (w), turns and stores a row's part; all lanes of a row take part.
  __device__ inline void finish(const Raw<8, T>& rx, const Raw<8, T>& ry, bool norm, const Raw<8, T>& wx, const Raw<8, T>& wy,
                                float eps, bool turn, T* dst, bool live) const {
    float x[8], y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) { x[i] = rx[i]; y[i] = ry[i]; }
    if (norm) {
      float sum = 0.0f;
#pragma unroll
      for (int i = 0; i < 8; ++i) sum += x[i] * x[i] + y[i] * y[i];
#pragma unroll
      for (int m = 1; m < U; m *= 2) sum += __shfl_xor(sum, m);
      const float r = 1.0f / sqrtf(sum * (1.0f / D) + eps);
#pragma unroll
      for (int i = 0; i < 8; ++i) { x[i] *= r * wx[i]; y[i] *= r * wy[i]; }
    }
    if (turn && turns) {
      if (!half) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float x0 = x[2 * i], y0 = y[2 * i];
          x[2 * i] = x0 * c[i] - x[2 * i + 1] * s[i];
          x[2 * i + 1] = x0 * s[i] + x[2 * i + 1] * c[i];
          y[2 * i] = y0 * c[4 + i] - y[2 * i + 1] * s[4 + i];
          y[2 * i + 1] = y0 * s[4 + i] + y[2 * i + 1] * c[4 + i];
        }
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float x0 = x[i];
          x[i] = x0 * c[i] - y[i] * s[i];
          y[i] = x0 * s[i] + y[i] * c[i];
        }
      }
    }
    if (live) {
      store8(dst + ca, x);
      store8(dst + cb, y);
    }
  }
};

// Few tokens: a workgroup to a token, its heads side by side in the lanes.  The
// lanes of a wavefront form each cosine and sine once (there are at most 64
// frequencies) and take their 8 from one another.  Latency bounds it: four rounds
// of loads, each with the address from the one before (a frequency's axis, its
// position, the pointers of the lane's head, the rows).  One token 3.2 us in the
// kernel, 2331 of 20 heads of width 64 in fp32 (23.9 MB) 9.2, half of a copy's
// rate, with 64% of the wavefronts' cycles waiting.
template <typename T, int D, int N>
__global__ __launch_bounds__(256) void rotate_token(RotateArgs<N> a) {
  constexpr int U = D / 16, HEADS = 64 / U;
  const RotateSeq& s = a.seq[blockIdx.y];
  const int lane = threadIdx.x & 63, wave = wave_id();
  const int64_t t = blockIdx.x;
  if (t >= s.n) return;
  Part<T, D> part(lane % U, a.rot, a.neighbours);
  floatx2 mine = floatx2{1.0f, 0.0f};
  if (lane < a.rot / 2) mine = turn_of(gload<int32_t>(s.pos + a.axis[lane] * s.pos_s + t), a.turns[lane]);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    part.c[i] = __shfl(mine[0], lane % U * 8 + i);
    part.s[i] = __shfl(mine[1], lane % U * 8 + i);
  }
  const int h_q = a.h_q, h_kv = a.h_kv;
  for (int h = wave * HEADS + lane / U; h < h_q + 2 * h_kv; h += 4 * HEADS) {
    const int kind = h < h_q ? 0 : h < h_q + h_kv ? 1 : 2;
    const int g = kind == 0 ? h : kind == 1 ? h - h_q : h - h_q - h_kv;
    const T* src = static_cast<const T*>(kind == 0 ? s.q : kind == 1 ? s.k : s.v) +
                   (kind == 0 ? g * s.q_hs + t * s.q_rs : g * s.kv_hs + t * s.kv_rs);
    T* dst = static_cast<T*>(kind == 0 ? s.q_out : kind == 1 ? s.k_out : s.v_out) +
             (kind == 0 ? g * s.qo_hs + t * s.qo_rs : g * s.o_hs + t * s.o_rs);
    const T* w = static_cast<const T*>(kind == 0 ? a.q_w : kind == 1 ? a.k_w : nullptr);
    Raw<8, T> x, y, wx = {}, wy = {};
    x.load(src + part.ca);
    y.load(src + part.cb);
    if (w) {
      wx.load(w + part.ca);
      wy.load(w + part.cb);
    }
    part.finish(x, y, w != nullptr, wx, wy, a.eps, kind != 2, dst, true);
  }
  if (s.mod && threadIdx.x == 0) s.mod_out[t] = gload<uint8_t>(s.mod + t);
}

// Many tokens: a workgroup to 1024 / D neighbouring tokens, a head of all of
// them to a wavefront at a time: what depends on the head is scalar, a token's
// cosines and sines are formed once (through LDS) and stay in registers, and
// the next head's rows are on their way while one is worked on.
// Bandwidth bounds it: 16384 tokens of 36 heads of width 128 (302 MB read and
// written) take 62 us, 4.9 TB/s, where a copy reaches 5.2; with a
// workgroup to a token, whose vector instructions bound it, 66 us.
template <typename T, int D, int N>
__global__ __launch_bounds__(256) void rotate_tokens(RotateArgs<N> a) {
  constexpr int U = D / 16, TOKENS = 64 / U, F = D / 2;
  const RotateSeq& s = a.seq[blockIdx.y];
  const int lane = threadIdx.x & 63, wave = wave_id();
  const int64_t t0 = (int64_t)blockIdx.x * TOKENS;
  if (t0 >= s.n) return;
  __shared__ floatx2 turn[TOKENS][F];
  for (int e = threadIdx.x; e < TOKENS * F; e += 256) {
    const int i = e / F, j = e % F;
    if (j < a.rot / 2 && t0 + i < s.n) turn[i][j] = turn_of(gload<int32_t>(s.pos + a.axis[j] * s.pos_s + t0 + i), a.turns[j]);
  }
  __syncthreads();
  const int tok = lane / U, u = lane % U;
  const bool live = t0 + tok < s.n;
  const int64_t t = min(t0 + tok, s.n - 1);
  Part<T, D> part(u, a.rot, a.neighbours);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const floatx2 y = part.turns && live ? turn[tok][u * 8 + i] : floatx2{1.0f, 0.0f};
    part.c[i] = y[0];
    part.s[i] = y[1];
  }
  const int h_q = a.h_q, h_kv = a.h_kv, heads = h_q + 2 * h_kv;
  const T* q_w = static_cast<const T*>(a.q_w);
  const T* k_w = static_cast<const T*>(a.k_w);
  Raw<8, T> qx = {}, qy = {}, kx = {}, ky = {}, x, y;
  if (q_w) { qx.load(q_w + part.ca); qy.load(q_w + part.cb); }
  if (k_w) { kx.load(k_w + part.ca); ky.load(k_w + part.cb); }
  const int64_t tq = t * s.q_rs, tkv = t * s.kv_rs, tqo = t * s.qo_rs, to = t * s.o_rs;
  const auto load = [&](int h) __attribute__((always_inline)) {
    const T* p = h < h_q ? static_cast<const T*>(s.q) + h * s.q_hs + tq
                         : static_cast<const T*>(h < h_q + h_kv ? s.k : s.v) + (h - h_q - (h < h_q + h_kv ? 0 : h_kv)) * s.kv_hs + tkv;
    x.load(p + part.ca);
    y.load(p + part.cb);
  };
  int h = wave;
  if (h < heads) load(h);
  for (; h < heads; h += 4) {
    const Raw<8, T> cx = x, cy = y;
    if (h + 4 < heads) load(h + 4);
    if (h < h_q)
      part.finish(cx, cy, q_w != nullptr, qx, qy, a.eps, true, static_cast<T*>(s.q_out) + h * s.qo_hs + tqo, live);
    else if (h < h_q + h_kv)
      part.finish(cx, cy, k_w != nullptr, kx, ky, a.eps, true, static_cast<T*>(s.k_out) + (h - h_q) * s.o_hs + to, live);
    else
      part.finish(cx, cy, false, kx, ky, a.eps, false, static_cast<T*>(s.v_out) + (h - h_q - h_kv) * s.o_hs + to, live);
  }
  if (s.mod && (int)threadIdx.x < TOKENS && t0 + threadIdx.x < s.n) s.mod_out[t0 + threadIdx.x] = gload<uint8_t>(s.mod + t0 + threadIdx.x);
}

template <typename T, int D>
void launch(const RotateArgs<kRotatesPerLaunch>& a, int n, int64_t rows, int64_t tokens, hipStream_t st) {
  // us, a workgroup to a token and to several, 36 heads of width 128: 2048 tokens 10.6 and 12.4, 4096 15.9 and 15.8,
  // 16384 66 and 62; 24 heads of fp32, width 64: 2048 8.0 and 9.9, 4096 11.9 and 11.5
  const bool many = tokens >= 4096;
  constexpr int TOKENS = 1024 / D;
  const dim3 grid((unsigned)(many ? (rows + TOKENS - 1) / TOKENS : rows), n);
  if (n == 1) {
    RotateArgs<1> one;
    one.seq[0] = a.seq[0];
    std::memcpy(one.turns, a.turns, sizeof a - offsetof(RotateArgs<kRotatesPerLaunch>, turns));
    if (many) rotate_tokens<T, D, 1><<<grid, 256, 0, st>>>(one);
    else rotate_token<T, D, 1><<<grid, 256, 0, st>>>(one);
  } else if (many) {
    rotate_tokens<T, D, kRotatesPerLaunch><<<grid, 256, 0, st>>>(a);
  } else {
    rotate_token<T, D, kRotatesPerLaunch><<<grid, 256, 0, st>>>(a);
  }
}

}  // namespace

hipError_t launch_rotate(const AttnDims& dm, const RotateArgs<kRotatesPerLaunch>& a, int n, hipStream_t st) {
  int64_t rows = 0, tokens = 0;
  for (int i = 0; i < n; ++i) {
    rows = std::max(rows, a.seq[i].n);
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
