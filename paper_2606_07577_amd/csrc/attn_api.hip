// Host side of the operators around the compression step: handle, argument
// checks, and descriptors into kernel arguments.
#include <new>

#include "attn_checks.h"

using namespace omnimem;

namespace {

omnimem_status check_held(omnimem_attn* attn, const omnimem_held& s, int i, bool pack) {
  const int H = attn->cfg.n_kv_heads;
  if (s.n_rows < 0 || s.n_rows > kMaxRows) return bad(attn, i, "n_rows out of range");
  if (s.n_rows == 0) return OMNIMEM_OK;
  const bool ok = pack ? readable(attn, s.k, H, s.n_rows, s.kv_head_stride, s.kv_row_stride) &&
                             readable(attn, s.v, H, s.n_rows, s.kv_head_stride, s.kv_row_stride)
                       : writable(attn, s.k, H, s.n_rows, s.kv_head_stride, s.kv_row_stride) &&
                             writable(attn, s.v, H, s.n_rows, s.kv_head_stride, s.kv_row_stride);
  if (!ok) return fail(attn, OMNIMEM_ERR_INVALID_ARG, "sequence %d: k and v %s", i, kStride);
  const int64_t bytes = omnimem_memory_bytes(attn->cfg.head_dim, s.n_rows);
  if (!s.data || !aligned(s.data, 16) || s.data_head_stride % 16 || s.data_head_stride < 0 ||
      s.data_head_stride >= kMaxSpan / 1024 || (H > 1 && s.data_head_stride < bytes))
    return bad(attn, i, "data must be given, 16-byte aligned, its head stride a multiple of 16, at least a head's bytes and below 64 GiB");
  const Span k = span(attn, s.k, H, s.n_rows, s.kv_head_stride, s.kv_row_stride);
  const Span v = span(attn, s.v, H, s.n_rows, s.kv_head_stride, s.kv_row_stride);
  const Span m = {reinterpret_cast<uintptr_t>(s.data), H, 1, s.data_head_stride, bytes, bytes};
  if (overlap(k, m) || overlap(v, m) || (!pack && overlap(k, v))) return bad(attn, i, "k, v and data overlap");
  return OMNIMEM_OK;
}

omnimem_status hold(omnimem_attn* attn, const omnimem_held* seqs, int32_t n, hipStream_t stream, bool pack) {
  omnimem_status st = begin(attn, seqs, n);
  if (st != OMNIMEM_OK) return st;
  for (int i = 0; i < n; ++i)
    if ((st = check_held(attn, seqs[i], i, pack)) != OMNIMEM_OK) return st;
  OnDevice dev(attn->device);
  hipError_t e = dev.err;
  for (int i0 = 0; i0 < n && e == hipSuccess; i0 += kHeldPerLaunch) {
    HeldArgs a;
    const int m = std::min(kHeldPerLaunch, n - i0);
    for (int i = 0; i < m; ++i) {
      const omnimem_held& s = seqs[i0 + i];
      a.seq[i] = {static_cast<char*>(s.k), static_cast<char*>(s.v), static_cast<char*>(s.data),
                  s.kv_head_stride, s.kv_row_stride, s.data_head_stride, s.n_rows};
    }
    e = launch_hold(attn->dm, a, m, pack, stream);
  }
  return done(attn, e, pack ? "omnimem_pack" : "omnimem_unpack");
}

}  // namespace

extern "C" {

omnimem_status omnimem_attn_create(const omnimem_attn_config* cfg, omnimem_attn** out) {
  if (!cfg || !out) return fail(nullptr, OMNIMEM_ERR_INVALID_ARG, "null argument");
  *out = nullptr;
  const omnimem_attn_config& c = *cfg;
  if (c.n_q_heads < 1 || c.n_kv_heads < 1 || c.n_q_heads % c.n_kv_heads != 0 || c.n_q_heads > 1024)
    return fail(nullptr, OMNIMEM_ERR_INVALID_ARG, "bad sizes: need 1 <= H_q <= 1024 and H_kv | H_q");
  if (c.head_dim != 64 && c.head_dim != 128)
    return fail(nullptr, OMNIMEM_ERR_UNSUPPORTED, "head_dim %d: supported 64 and 128", c.head_dim);
  if (c.dtype != OMNIMEM_BF16 && c.dtype != OMNIMEM_F32) return fail(nullptr, OMNIMEM_ERR_UNSUPPORTED, "dtype %d", c.dtype);
  omnimem_attn* attn = new (std::nothrow) omnimem_attn();
  if (!attn) return fail(nullptr, OMNIMEM_ERR_HIP, "out of host memory");
  attn->cfg = c;
  attn->dm = {c.n_q_heads, c.n_kv_heads, c.n_q_heads / c.n_kv_heads, c.head_dim, c.dtype};
  hipError_t e = hipGetDevice(&attn->device);
  if (e == hipSuccess) {
    int cus = 0;
    if (hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, attn->device) == hipSuccess && cus > 0)
      attn->compute_units = cus;
    e = hipMalloc(&attn->workspace, (size_t)kPartBytes + kMaxPartials * sizeof(int));
    if (e == hipSuccess) e = hipMemset(static_cast<char*>(attn->workspace) + kPartBytes, 0, kMaxPartials * sizeof(int));
    if (e == hipSuccess) e = hipDeviceSynchronize();          // (calls come on streams that do not wait for the null stream)
    if (e == hipSuccess) e = prepare_attend(attn->dm);
  }
  if (e != hipSuccess) {
    (void)hipGetLastError();
    (void)hipFree(attn->workspace);
    delete attn;
    return fail(nullptr, OMNIMEM_ERR_HIP, "workspace: %s", hipGetErrorString(e));
  }
  *out = attn;
  return OMNIMEM_OK;
}

omnimem_status omnimem_attn_destroy(omnimem_attn* attn) {
  if (!attn) return OMNIMEM_OK;
  {
    OnDevice dev(attn->device);
    (void)hipDeviceSynchronize();
    (void)hipFree(attn->workspace);
  }
  delete attn;
  return OMNIMEM_OK;
}

const char* omnimem_attn_last_error(const omnimem_attn* attn) { return attn ? attn->err : g_error; }

int64_t omnimem_memory_bytes(int32_t head_dim, int64_t rows) {
  if ((head_dim != 64 && head_dim != 128) || rows < 0 || rows > kMaxRows) return 0;
  return (rows + kMemRows - 1) / kMemRows * 34 * head_dim;
}

omnimem_status omnimem_rotate(omnimem_attn* attn, const omnimem_rope* rope, const omnimem_projection* seqs, int32_t n,
                              hipStream_t stream) {
  omnimem_status st = begin(attn, seqs, n);
  if (st != OMNIMEM_OK) return st;
  const omnimem_attn_config& c = attn->cfg;
  RotateArgs<kRotatesPerLaunch> a;
  if ((st = take_rope(attn, rope, a)) != OMNIMEM_OK) return st;
  for (int i = 0; i < n; ++i) {
    const omnimem_projection& s = seqs[i];
    if (s.n_rows < 0 || s.n_rows > kMaxRows) return bad(attn, i, "n_rows out of range");
    if (s.n_rows == 0) continue;
    if (!readable(attn, s.q, c.n_q_heads, s.n_rows, s.q_head_stride, s.q_row_stride) ||
        !readable(attn, s.k, c.n_kv_heads, s.n_rows, s.kv_head_stride, s.kv_row_stride) ||
        !readable(attn, s.v, c.n_kv_heads, s.n_rows, s.kv_head_stride, s.kv_row_stride))
      return fail(attn, OMNIMEM_ERR_INVALID_ARG, "sequence %d: q, k and v %s", i, kStride);
    if (!s.pos || !aligned(s.pos, 4) || s.pos_stride < 0 || s.pos_stride >= kMaxSpan / 16)
      return bad(attn, i, "pos must be given, 4-byte aligned, its stride >= 0 and below 2^42");
    if (!writable(attn, s.q_out, c.n_q_heads, s.n_rows, s.q_out_head_stride, s.q_out_row_stride) ||
        !writable(attn, s.k_out, c.n_kv_heads, s.n_rows, s.out_head_stride, s.out_row_stride) ||
        !writable(attn, s.v_out, c.n_kv_heads, s.n_rows, s.out_head_stride, s.out_row_stride))
      return fail(attn, OMNIMEM_ERR_INVALID_ARG, "sequence %d: q_out, k_out and v_out %s, no two rows on one place", i, kStride);
    if ((s.modality == nullptr) != (s.modality_out == nullptr))
      return bad(attn, i, "modality and modality_out must be given together");
    const Span in[3] = {span(attn, s.q, c.n_q_heads, s.n_rows, s.q_head_stride, s.q_row_stride),
                        span(attn, s.k, c.n_kv_heads, s.n_rows, s.kv_head_stride, s.kv_row_stride),
                        span(attn, s.v, c.n_kv_heads, s.n_rows, s.kv_head_stride, s.kv_row_stride)};
    const Span to[3] = {span(attn, s.q_out, c.n_q_heads, s.n_rows, s.q_out_head_stride, s.q_out_row_stride),
                        span(attn, s.k_out, c.n_kv_heads, s.n_rows, s.out_head_stride, s.out_row_stride),
                        span(attn, s.v_out, c.n_kv_heads, s.n_rows, s.out_head_stride, s.out_row_stride)};
    for (int x = 0; x < 3; ++x)
      for (int y = 0; y < 3; ++y)
        if ((x != y && overlap(to[x], to[y])) || (!(x == y && same(to[x], in[y])) && overlap(to[x], in[y])))
          return bad(attn, i, "an output overlaps another, or an input that it is not");
    const Span modality = {reinterpret_cast<uintptr_t>(s.modality), 1, 1, 0, 0, s.n_rows};
    const Span modality_out = {reinterpret_cast<uintptr_t>(s.modality_out), 1, 1, 0, 0, s.n_rows};
    const auto rows = [](const Span (&x)[3], const Span& y) { return overlap(x[0], y) || overlap(x[1], y) || overlap(x[2], y); };
    const auto written = [&](const Span& x) { return rows(to, x) || (s.modality && overlap(modality_out, x)); };
    if (beside_rows(attn, *rope, s, written)) return bad(attn, i, "an output overlaps pos or a norm's weights");
    if (s.modality && ((s.modality != s.modality_out && overlap(modality, modality_out)) || rows(to, modality) || rows(to, modality_out) ||
                       rows(in, modality_out)))
      return bad(attn, i, "modality or modality_out overlaps the other, or rows");
  }
  OnDevice dev(attn->device);
  hipError_t e = dev.err;
  for (int i0 = 0; i0 < n && e == hipSuccess; i0 += kRotatesPerLaunch) {
    const int m = std::min(kRotatesPerLaunch, n - i0);
    for (int i = 0; i < m; ++i) {
      const omnimem_projection& s = seqs[i0 + i];
      a.seq[i] = {s.q, s.k, s.v, s.pos, s.modality, s.q_out, s.k_out, s.v_out, s.modality_out,
                  s.q_head_stride, s.q_row_stride, s.kv_head_stride, s.kv_row_stride, s.pos_stride,
                  s.q_out_head_stride, s.q_out_row_stride, s.out_head_stride, s.out_row_stride, s.n_rows};
    }
    e = launch_rotate(attn->dm, a, m, stream);
  }
  return done(attn, e, "omnimem_rotate");
}

omnimem_status omnimem_pack(omnimem_attn* attn, const omnimem_held* seqs, int32_t n, hipStream_t stream) {
  return hold(attn, seqs, n, stream, true);
}

omnimem_status omnimem_unpack(omnimem_attn* attn, const omnimem_held* seqs, int32_t n, hipStream_t stream) {
  return hold(attn, seqs, n, stream, false);
}

omnimem_status omnimem_attend(omnimem_attn* attn, const omnimem_query* seqs, int32_t n, int32_t causal, hipStream_t stream) {
  omnimem_status st = begin(attn, seqs, n);
  if (st != OMNIMEM_OK) return st;
  const omnimem_attn_config& c = attn->cfg;
  const int Hq = c.n_q_heads, H = c.n_kv_heads;
  for (int i = 0; i < n; ++i) {
    const omnimem_query& s = seqs[i];
    if (s.n_queries < 0 || s.n_queries > kMaxRows / attn->dm.group || s.memory_rows < 0 ||
        s.memory_rows > kMaxRows || s.n_tail < 0 || s.n_tail > kMaxRows)
      return bad(attn, i, "n_queries, memory_rows or n_tail out of range");
    if (s.n_queries == 0) continue;
    if (!std::isfinite(log2_scale(s, c.head_dim))) return bad(attn, i, "sm_scale times log2(e) is not finite");
    if (!readable(attn, s.q, Hq, s.n_queries, s.q_head_stride, s.q_row_stride))
      return fail(attn, OMNIMEM_ERR_INVALID_ARG, "sequence %d: q %s", i, kStride);
    if (s.n_tail > 0 && (!readable(attn, s.k, H, s.n_tail, s.kv_head_stride, s.kv_row_stride) ||
                         !readable(attn, s.v, H, s.n_tail, s.kv_head_stride, s.kv_row_stride)))
      return fail(attn, OMNIMEM_ERR_INVALID_ARG, "sequence %d: k and v %s", i, kStride);
    if (s.n_tail > 0 && s.kv_row_stride * (int64_t)elt(attn) >= (int64_t)1 << 24)
      return bad(attn, i, "k and v need a row stride below 16 MiB");
    const int64_t bytes = omnimem_memory_bytes(c.head_dim, s.memory_rows);
    if (s.memory_rows > 0 && (!s.memory || !aligned(s.memory, 16) || s.memory_head_stride % 16 || s.memory_head_stride < 0 ||
                              s.memory_head_stride / 16 > UINT32_MAX ||
                              (H > 1 && s.memory_head_stride < bytes)))
      return bad(attn, i, "memory must be given, 16-byte aligned, its head stride a multiple of 16 and at least a head's bytes");
    if (!writable(attn, s.out, Hq, s.n_queries, s.out_head_stride, s.out_row_stride))
      return fail(attn, OMNIMEM_ERR_INVALID_ARG, "sequence %d: out %s, no two rows on one place", i, kStride);
    if (s.lse && (!aligned(s.lse, 4) || s.lse_head_stride < (Hq > 1 ? s.n_queries : 0) || s.lse_head_stride > UINT32_MAX))
      return bad(attn, i, "lse must be 4-byte aligned, its head stride at least n_queries and below 2^32");
    const Span q = span(attn, s.q, Hq, s.n_queries, s.q_head_stride, s.q_row_stride);
    const Span o = span(attn, s.out, Hq, s.n_queries, s.out_head_stride, s.out_row_stride);
    const Span lse = {reinterpret_cast<uintptr_t>(s.lse), Hq, 1, s.lse_head_stride * 4, s.n_queries * 4, s.n_queries * 4};
    const auto written = [&](const Span& x) { return overlap(o, x) || (s.lse && overlap(lse, x)); };
    bool clash = written(q) || (s.lse && overlap(o, lse));
    if (s.n_tail > 0)
      clash = clash || written(span(attn, s.k, H, s.n_tail, s.kv_head_stride, s.kv_row_stride)) ||
              written(span(attn, s.v, H, s.n_tail, s.kv_head_stride, s.kv_row_stride));
    if (s.memory_rows > 0)
      clash = clash || written({reinterpret_cast<uintptr_t>(s.memory), H, 1, s.memory_head_stride, bytes, bytes});
    if (clash) return bad(attn, i, "out or lse overlaps the other, q, k, v or the memory");
  }
  OnDevice dev(attn->device);
  hipError_t e = dev.err;
  const int64_t per = 16 / (int64_t)elt(attn);
  const auto units = [per](int64_t stride) { return (uint32_t)(stride / per); };
  for (int i0 = 0; i0 < n && e == hipSuccess;) {
    AttendArgs<kQueriesPerLaunch> a;
    a.causal = causal ? 1 : 0;
    int m = 0;
    for (; i0 < n && m < kQueriesPerLaunch; ++i0) {
      const omnimem_query& s = seqs[i0];
      if (s.n_queries == 0) continue;
      QuerySeq& x = a.seq[m++];
      x.q = s.q; x.mem = static_cast<const char*>(s.memory); x.k = s.k; x.v = s.v; x.out = s.out; x.lse = s.lse;
      x.q_hs = units(s.q_head_stride); x.q_rs = units(s.q_row_stride);
      x.kv_hs = units(s.kv_head_stride); x.kv_rs = units(s.kv_row_stride);
      x.out_hs = units(s.out_head_stride); x.out_rs = units(s.out_row_stride);
      x.mem_hs = (uint32_t)(s.memory_head_stride / 16); x.lse_hs = (uint32_t)s.lse_head_stride;
      x.scale_log2 = log2_scale(s, c.head_dim);
      x.nq = (int32_t)s.n_queries; x.nm = (int32_t)s.memory_rows; x.nt = (int32_t)s.n_tail;
    }
    if (m) e = launch_attend(attn->dm, a, m, attn->compute_units, attn->workspace, stream);
  }
  return done(attn, e, "omnimem_attend");
}

}  // extern "C"
