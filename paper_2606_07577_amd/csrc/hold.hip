// Kept rows in 4 bits: packing rows into a memory's blocks and bringing them
// back.
#include "../../include/omnimem.h"
#include "attn.h"

namespace omnimem {
namespace {

// The scale byte of a group whose largest magnitude has the bits m: the
// smallest exponent with m <= 1.75 * 2^(e + 2), from the exponent field of m
// with anything past 1.75 carried into it; 2^125 at most, whose largest code
// is 6 * 2^125 (a code of 4 * 2^126 would come back as an infinity).
__device__ inline uint32_t scale_byte(uint32_t m) {
  if (m >= 0x7F800000u) return kScaleNan;
  const int e = (int)((m + 0x1FFFFFu) >> 23) - 2;
  return (uint32_t)min(max(e, (int)kScaleMin), (int)kScaleMax);
}
__device__ inline uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }

// Eight values over the scale, each the nearest code (ties to even; the
// conversion takes what lies past 6 to 6), the first in the lowest bits.
__device__ inline uint32_t codes8(const float (&x)[8], uint32_t byte) {
  if (byte == kScaleNan) return 0;
  const float s = scale_of(byte);
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], s, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], s, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], s, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], s, 3);
  return w;
}

// One wavefront per block of 32 rows, whole rows read 16 bytes (d = 64: 8) a
// lane.  K: four lanes to a group of 32 channels, 8 channels each.  V: lane
// (i, g) has D/16 channels of rows 8 g .. 8 g + 7, a word of codes of each; the
// four lanes g agree on a channel's scale.  Bandwidth bounds both directions: 28
// layers of 4 heads of 4096 rows of width 128 (297 MB each way) are packed in
// 76 us, 3.9 TB/s, and unpacked in 49, 6.1 TB/s (a copy reaches 5.2; codes in
// whole lines through LDS: 78).  The packed rows go out as words of 32 lines.
template <typename T, int D>
__global__ __launch_bounds__(256) void pack_rows(HeldArgs a) {
  using B = MemBlock<D>;
  constexpr int C = D / 16;
  const HeldSeq& s = a.seq[blockIdx.z];
  const int lane = threadIdx.x & 63, g = lane >> 4, c0 = (lane & 15) * C;
  const int64_t block = (int64_t)blockIdx.x * 4 + wave_id();
  if (block * kMemRows >= s.n) return;
  const int valid = (int)min((int64_t)kMemRows, s.n - block * kMemRows);
  const T* k = reinterpret_cast<const T*>(s.k) + blockIdx.y * s.kv_hs + block * kMemRows * s.kv_rs;
  const T* v = reinterpret_cast<const T*>(s.v) + blockIdx.y * s.kv_hs + block * kMemRows * s.kv_rs;
  char* out = s.data + blockIdx.y * s.data_hs + block * B::BYTES;
  Raw<C, T> vr[8];
  Raw<8, T> kr[D / 16];
#pragma unroll
  for (int it = 0; it < D / 16; ++it) {
    const int slot = it * 64 + lane;
    kr[it].load(k + min(slot / (D / 8), valid - 1) * s.kv_rs + slot % (D / 8) * 8);
  }
#pragma unroll
  for (int r = 0; r < 8; ++r) vr[r].load(v + min(g * 8 + r, valid - 1) * s.kv_rs + c0);
  asm volatile("" ::: "memory");           // (every load is on its way before the first is waited for)
#pragma unroll
  for (int it = 0; it < D / 16; ++it) {
    const int slot = it * 64 + lane, t = slot / (D / 8), c8 = slot % (D / 8);
    float x[8];
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      x[i] = t < valid ? kr[it][i] : 0.0f;
      m = max(m, magnitude(x[i]));
    }
    m = max(m, (uint32_t)__shfl_xor((int)m, 1));
    m = max(m, (uint32_t)__shfl_xor((int)m, 2));
    const uint32_t byte = scale_byte(m);
    *reinterpret_cast<uint32_t*>(out + t * (D / 2) + c8 * 4) = codes8(x, byte);
    if ((c8 & 3) == 0) out[B::k_scale(t, c8 >> 2)] = (char)byte;
  }
#pragma unroll
  for (int i = 0; i < C; ++i) {
    float x[8];
    uint32_t m = 0;
#pragma unroll
    for (int r = 0; r < 8; ++r) {
      x[r] = g * 8 + r < valid ? vr[r][i] : 0.0f;
      m = max(m, magnitude(x[r]));
    }
    m = max(m, (uint32_t)__shfl_xor((int)m, 16));
    m = max(m, (uint32_t)__shfl_xor((int)m, 32));
    const uint32_t byte = scale_byte(m);
    *reinterpret_cast<uint32_t*>(out + B::V + (c0 + i) * 16 + g * 4) = codes8(x, byte);
    if (g == i * 4 / C) out[B::v_scale(c0 + i)] = (char)byte;
  }
}

template <int CPL>
__device__ inline void store_channels(uint16_t* p, const float (&x)[CPL]) {
  if constexpr (CPL == 1) *p = (uint16_t)round2(x[0], 0.0f);
  else *reinterpret_cast<uint32_t*>(p) = round2(x[0], x[1]);
}
template <int CPL>
__device__ inline void store_channels(float* p, const float (&x)[CPL]) {
#pragma unroll
  for (int i = 0; i < CPL; ++i) p[i] = x[i];
}
__device__ inline void store_values(uint16_t* p, uint32_t w, uint32_t byte) {
  *reinterpret_cast<uint4*>(p) = values8_bf16(w, scale_of(byte));
}
__device__ inline void store_values(float* p, uint32_t w, uint32_t byte) {
  float x[8];
  values8(w, byte, x);
  *reinterpret_cast<floatx4*>(p) = floatx4{x[0], x[1], x[2], x[3]};
  *reinterpret_cast<floatx4*>(p + 4) = floatx4{x[4], x[5], x[6], x[7]};
}

// The same the other way.
template <typename T, int D>
__global__ __launch_bounds__(256) void unpack_rows(HeldArgs a) {
  using B = MemBlock<D>;
  constexpr int CPL = D / 64;
  const HeldSeq& s = a.seq[blockIdx.z];
  const int lane = threadIdx.x & 63;
  const int64_t block = (int64_t)blockIdx.x * 4 + wave_id();
  if (block * kMemRows >= s.n) return;
  const int valid = (int)min((int64_t)kMemRows, s.n - block * kMemRows);
  T* k = reinterpret_cast<T*>(s.k) + blockIdx.y * s.kv_hs + block * kMemRows * s.kv_rs;
  T* v = reinterpret_cast<T*>(s.v) + blockIdx.y * s.kv_hs + block * kMemRows * s.kv_rs;
  const char* in = s.data + blockIdx.y * s.data_hs + block * B::BYTES;
  uint4 codes[CPL];
  uint32_t byte[CPL];
#pragma unroll
  for (int i = 0; i < CPL; ++i) {
    codes[i] = gload16(in + B::V + (lane * CPL + i) * 16);
    byte[i] = gload<uint8_t>(in + B::v_scale(lane * CPL + i));
  }
#pragma unroll
  for (int it = 0; it < D / 16; ++it) {
    const int slot = it * 64 + lane, t = slot / (D / 8), c8 = slot % (D / 8);
    const uint32_t w = gload<uint32_t>(in + t * (D / 2) + c8 * 4);
    const uint32_t b = gload<uint8_t>(in + B::k_scale(t, c8 >> 2));
    if (t < valid) store_values(k + t * s.kv_rs + c8 * 8, w, b);
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    float x[CPL][8];
#pragma unroll
    for (int i = 0; i < CPL; ++i) values8(j == 0 ? codes[i].x : j == 1 ? codes[i].y : j == 2 ? codes[i].z : codes[i].w, byte[i], x[i]);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float y[CPL];
#pragma unroll
      for (int i = 0; i < CPL; ++i) y[i] = x[i][e];
      if (8 * j + e < valid) store_channels<CPL>(v + (8 * j + e) * s.kv_rs + lane * CPL, y);
    }
  }
}

template <typename T, int D>
void launch(const HeldArgs& a, dim3 grid, bool pack, hipStream_t st) {
  if (pack) pack_rows<T, D><<<grid, 256, 0, st>>>(a); else unpack_rows<T, D><<<grid, 256, 0, st>>>(a);
}

}  // namespace

hipError_t launch_hold(const AttnDims& dm, const HeldArgs& a, int n, bool pack, hipStream_t st) {
  int64_t rows = 0;
  for (int i = 0; i < n; ++i) rows = std::max(rows, a.seq[i].n);
  if (rows == 0) return hipSuccess;
  const dim3 grid((unsigned)((rows + 4 * kMemRows - 1) / (4 * kMemRows)), dm.h_kv, n);
  if (dm.dtype == OMNIMEM_BF16) {
    if (dm.d == 128) launch<uint16_t, 128>(a, grid, pack, st); else launch<uint16_t, 64>(a, grid, pack, st);
  } else {
    if (dm.d == 128) launch<float, 128>(a, grid, pack, st); else launch<float, 64>(a, grid, pack, st);
  }
  return hipGetLastError();
}

}  // namespace omnimem
