// A lane's share of a row's norm and rotation.
#pragma once

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
__device__ inline void store8(float* p, const float (&x)[4]) { *reinterpret_cast<floatx4*>(p) = floatx4{x[0], x[1], x[2], x[3]}; }

// Cosine and sine of a position times a frequency in turns, formed and reduced
// in 64 bits.
__device__ inline floatx2 turn_of(int32_t pos, double turns) {
  const double x = (double)pos * turns;
  float c, s;
  sincospif(2.0f * (float)(x - rint(x)), &s, &c);
  return floatx2{c, s};
}

// A lane's 2 C channels of a row: two runs of C that turn with C frequencies
// (against each other, or neighbours within them), D / 2C lanes to a row.
template <typename T, int D, int C = 8>
struct Part {
  static constexpr int U = D / (2 * C);
  int ca, cb;                // first channels of the runs
  bool turns, half;
  float c[C], s[C];
  __device__ inline Part(int u, int rot, int neighbours) {
    turns = u < rot / (2 * C);
    half = turns && !neighbours;
    ca = half ? C * u : 2 * C * u;
    cb = half ? rot / 2 + C * u : 2 * C * u + C;
  }
  // Normalises (w), turns and stores a row's part; all lanes of a row take part.
  __device__ inline void finish(const Raw<C, T>& rx, const Raw<C, T>& ry, bool norm, const Raw<C, T>& wx, const Raw<C, T>& wy,
                                float eps, bool turn, T* dst, bool live) const {
    float x[C], y[C];
#pragma unroll
    for (int i = 0; i < C; ++i) { x[i] = rx[i]; y[i] = ry[i]; }
    if (norm) {
      float sum = 0.0f;
#pragma unroll
      for (int i = 0; i < C; ++i) sum += x[i] * x[i] + y[i] * y[i];
#pragma unroll
      for (int m = 1; m < U; m *= 2) sum += __shfl_xor(sum, m);
      const float r = 1.0f / sqrtf(sum * (1.0f / D) + eps);
#pragma unroll
      for (int i = 0; i < C; ++i) { x[i] *= r * wx[i]; y[i] *= r * wy[i]; }
    }
    if (turn && turns) {
      if (!half) {
#pragma unroll
        for (int i = 0; i < C / 2; ++i) {
          const float x0 = x[2 * i], y0 = y[2 * i];
          x[2 * i] = x0 * c[i] - x[2 * i + 1] * s[i];
          x[2 * i + 1] = x0 * s[i] + x[2 * i + 1] * c[i];
          y[2 * i] = y0 * c[C / 2 + i] - y[2 * i + 1] * s[C / 2 + i];
          y[2 * i + 1] = y0 * s[C / 2 + i] + y[2 * i + 1] * c[C / 2 + i];
        }
      } else {
#pragma unroll
        for (int i = 0; i < C; ++i) {
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

}  // namespace
}  // namespace omnimem
