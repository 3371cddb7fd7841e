// What the host side of the operators around the compression step shares: the
// handle, its errors, and the checks of arrays.
#pragma once

#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "../../include/omnimem.h"
#include "attn.h"

struct omnimem_attn {
  omnimem_attn_config cfg;
  omnimem::AttnDims dm;
  int device = 0;
  int compute_units = 256;
  void* workspace = nullptr;
  char err[512] = "";
};

namespace omnimem {

inline thread_local char g_error[512] = "";    // of calls without a handle

namespace {

omnimem_status fail(omnimem_attn* attn, omnimem_status st, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(attn ? attn->err : g_error, sizeof g_error, fmt, ap);
  va_end(ap);
  return st;
}

omnimem_status bad(omnimem_attn* attn, int i, const char* what) {
  return fail(attn, OMNIMEM_ERR_INVALID_ARG, "sequence %d: %s", i, what);
}

// The handle's device is current for the call, the caller's again after it.
struct OnDevice {
  int before = -1, device;
  hipError_t err;
  explicit OnDevice(int d) : device(d) {
    err = hipGetDevice(&before);
    if (err == hipSuccess && before != d) err = hipSetDevice(d);
  }
  ~OnDevice() {
    if (before >= 0 && before != device) (void)hipSetDevice(before);
  }
};

constexpr int64_t kMaxRows = (int64_t)1 << 30;

size_t elt(const omnimem_attn* attn) { return attn->cfg.dtype == OMNIMEM_BF16 ? 2 : 4; }
bool aligned(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

// A strided [heads][rows][width] array, in bytes.
struct Span {
  uintptr_t base;
  int64_t heads, rows, hs, rs, width;
  uintptr_t end() const { return base + (uintptr_t)((heads - 1) * hs + (rows - 1) * rs + width); }
};
Span span(const omnimem_attn* a, const void* p, int64_t heads, int64_t rows, int64_t hs, int64_t rs) {
  const int64_t e = (int64_t)elt(a);
  return {reinterpret_cast<uintptr_t>(p), heads, rows, hs * e, rs * e, a->cfg.head_dim * e};
}
// Windows [0, w) and [off, off + v) of every period, off taken modulo it.
bool apart(int64_t period, int64_t w, int64_t v, int64_t off) {
  if (period <= 0) return false;
  off = ((off % period) + period) % period;
  return w <= off && off + v <= period;
}
// Whether two arrays can share a byte: not if their ranges are apart, nor if
// they are windows of the same rows (a fused projection's queries and keys)
// or of the same heads (two runs of rows of a cache).
bool overlap(const Span& a, const Span& b) {
  if (a.base >= b.end() || b.base >= a.end()) return false;
  const int64_t off = (int64_t)(b.base - a.base);
  if (a.rs == b.rs && apart(a.rs, (a.heads - 1) * a.hs + a.width, (b.heads - 1) * b.hs + b.width, off)) return false;
  if (a.hs == b.hs && apart(a.hs, (a.rows - 1) * a.rs + a.width, (b.rows - 1) * b.rs + b.width, off)) return false;
  return true;
}
bool same(const Span& a, const Span& b) { return a.base == b.base && (a.hs == b.hs || a.heads == 1) && (a.rs == b.rs || a.rows == 1); }
// Rows that are read: strides of 16-byte units below 64 GiB, rows of at least
// d, and no array past 64 TiB (sums of products of strides fit 64 bits).
constexpr int64_t kMaxSpan = (int64_t)1 << 46;
bool readable(const omnimem_attn* a, const void* p, int64_t heads, int64_t rows, int64_t hs, int64_t rs) {
  const int64_t e = (int64_t)elt(a);
  return p && aligned(p, 16) && hs >= 0 && rs >= a->cfg.head_dim && hs % (16 / e) == 0 && rs % (16 / e) == 0 &&
         hs / (16 / e) <= UINT32_MAX && rs / (16 / e) <= UINT32_MAX &&
         (double)(heads - 1) * (double)hs + (double)(rows - 1) * (double)rs < (double)(kMaxSpan / e);
}
// Rows that are written: each row of each head has its own place.
bool writable(const omnimem_attn* a, const void* p, int64_t heads, int64_t rows, int64_t hs, int64_t rs) {
  const int64_t d = a->cfg.head_dim;
  if (!readable(a, p, heads, rows, hs, rs)) return false;
  return heads == 1 || hs >= (rows - 1) * rs + d || (hs >= d && rs >= (heads - 1) * hs + d);
}

const char* kStride = "must be given, 16-byte aligned, strides of whole 16-byte units, row stride >= head_dim, all below 64 TiB";

omnimem_status begin(omnimem_attn* attn, const void* seqs, int32_t n) {
  if (!attn) return fail(nullptr, OMNIMEM_ERR_INVALID_ARG, "null handle");
  if (n < 0 || (n > 0 && !seqs)) return fail(attn, OMNIMEM_ERR_INVALID_ARG, "null sequences, or n < 0");
  return OMNIMEM_OK;
}

omnimem_status done(omnimem_attn* attn, hipError_t e, const char* what) {
  if (e != hipSuccess) return fail(attn, OMNIMEM_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
  attn->err[0] = 0;
  return OMNIMEM_OK;
}

// A rope's checks and its part of the kernels' arguments.
template <class Args>
omnimem_status take_rope(omnimem_attn* attn, const omnimem_rope* rope, Args& a) {
  const omnimem_attn_config& c = attn->cfg;
  if (!rope) return fail(attn, OMNIMEM_ERR_INVALID_ARG, "null rope");
  const omnimem_rope& r = *rope;
  if (r.rotary_dim < 0 || r.rotary_dim > c.head_dim || r.n_axes < 1 || r.n_axes > 4 || (r.rotary_dim > 0 && !r.inv_freq))
    return fail(attn, OMNIMEM_ERR_INVALID_ARG, "rope: need 0 <= rotary_dim <= head_dim, 1 to 4 axes, and inv_freq");
  if (r.rotary_dim % 16) return fail(attn, OMNIMEM_ERR_UNSUPPORTED, "rotary_dim %d: supported multiples of 16", r.rotary_dim);
  if (!std::isfinite(r.eps) || r.eps < 0.0f) return fail(attn, OMNIMEM_ERR_INVALID_ARG, "rope: eps must be finite and >= 0");
  if (!aligned(r.q_weight, 16) || !aligned(r.k_weight, 16))
    return fail(attn, OMNIMEM_ERR_INVALID_ARG, "rope: weights must be 16-byte aligned");
  for (int j = 0; j < r.rotary_dim / 2; ++j) {
    const double f = r.inv_freq[j];
    if (!std::isfinite(f) || (r.axis && r.axis[j] >= r.n_axes))
      return fail(attn, OMNIMEM_ERR_INVALID_ARG, "rope: frequency %d is not finite, or its axis is not below n_axes", j);
    a.turns[j] = f / 6.283185307179586476925286766559;
    a.axis[j] = r.axis ? r.axis[j] : 0;
  }
  a.q_w = r.q_weight; a.k_w = r.k_weight;
  a.eps = r.eps; a.rot = r.rotary_dim; a.neighbours = r.neighbours ? 1 : 0;
  a.h_q = c.n_q_heads; a.h_kv = c.n_kv_heads;
  return OMNIMEM_OK;
}

// Whether a sequence's rotation reads positions, or a norm's weights, that are
// `written`.
template <class Seq, class Written>
bool beside_rows(const omnimem_attn* a, const omnimem_rope& r, const Seq& s, Written&& written) {
  const auto array = [](const void* p, int64_t n, int64_t stride, int64_t bytes) {
    return Span{reinterpret_cast<uintptr_t>(p), n, 1, stride, 0, bytes};
  };
  const int64_t width = a->cfg.head_dim * (int64_t)elt(a);
  return written(array(s.pos, r.n_axes, s.pos_stride * 4, s.n_rows * 4)) || (r.q_weight && written(array(r.q_weight, 1, 0, width))) ||
         (r.k_weight && written(array(r.k_weight, 1, 0, width)));
}

template <class Query>
float log2_scale(const Query& s, int d) {
  return (float)((s.sm_scale != 0.0f ? (double)s.sm_scale : 1.0 / std::sqrt((double)d)) * 1.4426950408889634);
}

}  // namespace
}  // namespace omnimem
