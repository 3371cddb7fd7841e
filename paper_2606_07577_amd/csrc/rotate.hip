// A chunk's projected rows to their places behind the cache: per-head norm
// and rotation of queries and keys, values copied, in one pass.
#include <cstddef>
#include <cstring>

#include "../../include/omnimem.h"
#include "attn.h"

namespace omnimem {
namespace {

// Eight consecutive elements of a row, as fp32.
__device__ inline void load8(const uint16_t* p, float (&x)[8]) {
  const uint4 w = gload16(p);
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(u[i] << 16);
    x[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u);
  }
}
__device__ inline void load8(const float* p, float (&x)[8]) {
  const floatx4 a = gload<floatx4>(p), b = gload<floatx4>(p + 4);
#pragma unroll
  for (int i = 0; i < 4; ++i) { x[i] = a[i]; x[4 + i] = b[i]; }
}
__device__ inline void store8(uint16_t* p, const float (&x)[8]) {
  *reinterpret_cast<uint4*>(p) = make_uint4(round2(x[0], x[1]), round2(x[2], x[3]), round2(x[4], x[5]), round2(x[6], x[7]));
}
__device__ inline void store8(float* p, const float (&x)[8]) {
  *reinterpret_cast<floatx4*>(p) = floatx4{x[0], x[1], x[2], x[3]};
  *reinterpret_cast<floatx4*>(p + 4) = floatx4{x[4], x[5], x[6], x[7]};
}

// A workgroup takes a token.  A lane holds a head's 16 channels that turn with
// 8 frequencies: two runs of 8, D/16 lanes to a head.  The lanes of a wavefront
// form each of the token's cosines and sines once (there are at most 64
// frequencies) and take their 8 from one another; they serve all its heads.
// Bandwidth bounds it: 16384 tokens of 36 heads of width 128 (302 MB read and
// written) take 66 us, 4.6 TB/s, where a copy reaches 5.2; a wavefront to a
// token, or four tokens to a workgroup, take 66 to 70.
template <typename T, int D, int N>
__global__ __launch_bounds__(256) void rotate_rows(RotateArgs<N> a) {
  constexpr int U = D / 16, HEADS = 64 / U;
  const RotateSeq& s = a.seq[blockIdx.y];
  const int lane = threadIdx.x & 63, wave = wave_id();
  const int64_t t = blockIdx.x;
  if (t >= s.n) return;
  const int rot = a.rot, u = lane % U;
  const bool turns = u < rot / 16;
  float c = 1.0f, sn = 0.0f;
  if (lane < rot / 2) {
    const int32_t p = gload<int32_t>(s.pos + a.axis[lane] * s.pos_s + t);
    const double x = (double)p * a.turns[lane];
    const float f = (float)(x - rint(x));   // of a turn
    sincospif(2.0f * f, &sn, &c);
  }
  float cs[8], sns[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    cs[i] = __shfl(c, u * 8 + i);
    sns[i] = __shfl(sn, u * 8 + i);
  }
  const bool half = turns && !a.neighbours;
  const int ca = half ? 8 * u : 16 * u, cb = half ? rot / 2 + 8 * u : 16 * u + 8;
  const int h_q = a.h_q, h_kv = a.h_kv;
  for (int h = wave * HEADS + lane / U; h < h_q + 2 * h_kv; h += 4 * HEADS) {
    const int kind = h < h_q ? 0 : h < h_q + h_kv ? 1 : 2;
    const int g = kind == 0 ? h : kind == 1 ? h - h_q : h - h_q - h_kv;
    const T* src = static_cast<const T*>(kind == 0 ? s.q : kind == 1 ? s.k : s.v) +
                   (kind == 0 ? g * s.q_hs + t * s.q_rs : g * s.kv_hs + t * s.kv_rs);
    T* dst = static_cast<T*>(kind == 0 ? s.q_out : kind == 1 ? s.k_out : s.v_out) +
             (kind == 0 ? g * s.qo_hs + t * s.qo_rs : g * s.o_hs + t * s.o_rs);
    float x[8], y[8];
    load8(src + ca, x);
    load8(src + cb, y);
    const T* w = static_cast<const T*>(kind == 0 ? a.q_w : kind == 1 ? a.k_w : nullptr);
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) sum += x[i] * x[i] + y[i] * y[i];
#pragma unroll
    for (int m = 1; m < U; m *= 2) sum += __shfl_xor(sum, m);
    if (w) {
      const float r = 1.0f / sqrtf(sum * (1.0f / D) + a.eps);
      float wx[8], wy[8];
      load8(w + ca, wx);
      load8(w + cb, wy);
#pragma unroll
      for (int i = 0; i < 8; ++i) { x[i] *= r * wx[i]; y[i] *= r * wy[i]; }
    }
    if (turns && kind != 2) {
      if (a.neighbours) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float x0 = x[2 * i], y0 = y[2 * i];
          x[2 * i] = x0 * cs[i] - x[2 * i + 1] * sns[i];
          x[2 * i + 1] = x0 * sns[i] + x[2 * i + 1] * cs[i];
          y[2 * i] = y0 * cs[4 + i] - y[2 * i + 1] * sns[4 + i];
          y[2 * i + 1] = y0 * sns[4 + i] + y[2 * i + 1] * cs[4 + i];
        }
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float x0 = x[i];
          x[i] = x0 * cs[i] - y[i] * sns[i];
          y[i] = x0 * sns[i] + y[i] * cs[i];
        }
      }
    }
    store8(dst + ca, x);
    store8(dst + cb, y);
  }
  if (s.mod && threadIdx.x == 0) s.mod_out[t] = gload<uint8_t>(s.mod + t);
}

template <typename T, int D>
void launch(const RotateArgs<kRotatesPerLaunch>& a, int n, int64_t rows, hipStream_t st) {
  if (n == 1) {
    RotateArgs<1> one;
    one.seq[0] = a.seq[0];
    std::memcpy(one.turns, a.turns, sizeof a - offsetof(RotateArgs<kRotatesPerLaunch>, turns));
    rotate_rows<T, D, 1><<<dim3((unsigned)rows, n), 256, 0, st>>>(one);
  } else {
    rotate_rows<T, D, kRotatesPerLaunch><<<dim3((unsigned)rows, n), 256, 0, st>>>(a);
  }
}

}  // namespace

hipError_t launch_rotate(const AttnDims& dm, const RotateArgs<kRotatesPerLaunch>& a, int n, hipStream_t st) {
  int64_t rows = 0;
  for (int i = 0; i < n; ++i) rows = std::max(rows, a.seq[i].n);
  if (rows == 0) return hipSuccess;
  if (dm.dtype == OMNIMEM_BF16) {
    if (dm.d == 128) launch<uint16_t, 128>(a, n, rows, st); else launch<uint16_t, 64>(a, n, rows, st);
  } else {
    if (dm.d == 128) launch<float, 128>(a, n, rows, st); else launch<float, 64>(a, n, rows, st);
  }
  return hipGetLastError();
}

}  // namespace omnimem
