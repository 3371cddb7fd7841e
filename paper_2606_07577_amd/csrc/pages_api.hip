// Host side of the operators on caches in pages: argument checks, and
// descriptors into kernel arguments.
#include "attn_checks.h"

using namespace omnimem;

namespace {

// A store's checks and its part of the kernels' arguments; its K and V as
// arrays (pages for heads), and their axes from the innermost out, in bytes.
struct Axis {
  int64_t count, stride;
};
struct Store {
  PagePool pool;
  Span k, v;
  Axis axes[3];
  int64_t width, extent;
};
// Whether K or V of two such stores, `off` bytes apart, share a byte.  An axis
// begins where the one inside it ends, so of its steps only the two next to
// `off` come near enough.
bool meet(const Store& x, int64_t off, int n = 3) {
  if (off < 0) off = -off;
  if (n == 0) return off < x.width;
  if (n == 3 && off >= x.extent) return false;
  const Axis& a = x.axes[n - 1];
  if (a.count == 1) return meet(x, off, n - 1);
  for (int64_t i = off / a.stride; i <= off / a.stride + 1 && i < a.count; ++i)
    if (meet(x, off - i * a.stride, n - 1)) return true;
  return false;
}
// The bytes from the first to the last of some stores' K or V.
struct Range {
  uintptr_t lo = UINTPTR_MAX, hi = 0;
  bool apart(const void* p, int64_t extent) const {
    const uintptr_t at = reinterpret_cast<uintptr_t>(p);
    return at >= hi || at + (uintptr_t)extent <= lo;
  }
  void add(const void* p, int64_t extent) {
    const uintptr_t at = reinterpret_cast<uintptr_t>(p);
    lo = std::min(lo, at);
    hi = std::max(hi, at + (uintptr_t)extent);
  }
};
int64_t apart_by(const void* a, const void* b) { return static_cast<const char*>(b) - static_cast<const char*>(a); }
omnimem_status take_pages(omnimem_attn* attn, const omnimem_pages* pages, Store& x) {
  if (!pages) return fail(attn, OMNIMEM_ERR_INVALID_ARG, "null pages");
  const omnimem_pages& p = *pages;
  const int64_t e = (int64_t)elt(attn), d = attn->cfg.head_dim;
  int shift = 4;
  while (shift < 8 && 1 << shift != p.page_rows) ++shift;
  if (1 << shift != p.page_rows)
    return fail(attn, OMNIMEM_ERR_UNSUPPORTED, "page_rows %d: supported 16, 32, 64, 128 and 256", p.page_rows);
  if (p.n_pages < 1 || !p.k || !p.v || !aligned(p.k, 16) || !aligned(p.v, 16))
    return fail(attn, OMNIMEM_ERR_INVALID_ARG, "pages: need 1 page at least, and k and v, 16-byte aligned");
  // the three axes from the innermost out: each begins where the one inside it ends
  Axis axes[3] = {{p.page_rows, p.row_stride}, {attn->cfg.n_kv_heads, p.head_stride}, {p.n_pages, p.page_stride}};
  std::sort(axes, axes + 3, [](const Axis& a, const Axis& b) { return a.stride < b.stride || (a.stride == b.stride && a.count < b.count); });
  int64_t extent = d;
  double bytes = (double)d * e;
  for (const Axis& a : axes) {
    if (a.stride < 0 || a.stride % (16 / e) || a.stride >= kMaxSpan / e)
      return fail(attn, OMNIMEM_ERR_INVALID_ARG, "pages: strides must be whole 16-byte units, >= 0 and below 64 TiB");
    if (a.count == 1) continue;
    bytes += (double)(a.count - 1) * (double)a.stride * e;
    if (a.stride < extent || bytes >= (double)kMaxSpan)
      return fail(attn, OMNIMEM_ERR_INVALID_ARG, "pages: rows lie on one another, or span 64 TiB");
    extent += (a.count - 1) * a.stride;
  }
  if (p.row_stride * e >= (int64_t)1 << 24) return fail(attn, OMNIMEM_ERR_INVALID_ARG, "pages: need a row stride below 16 MiB");
  const int64_t page = ((p.page_rows - 1) * p.row_stride + (attn->cfg.n_kv_heads - 1) * p.head_stride + d) * e;
  x.pool = {static_cast<char*>(p.k), static_cast<char*>(p.v), p.page_stride * e, p.head_stride * e,
            (uint32_t)(p.row_stride * e), (uint32_t)p.n_pages, shift};
  x.k = {reinterpret_cast<uintptr_t>(p.k), p.n_pages, 1, p.page_stride * e, 0, page};
  x.v = {reinterpret_cast<uintptr_t>(p.v), p.n_pages, 1, p.page_stride * e, 0, page};
  for (int i = 0; i < 3; ++i) x.axes[i] = {axes[i].count, axes[i].stride * e};
  x.width = d * e;
  x.extent = extent * e;
  if (meet(x, apart_by(p.k, p.v))) return fail(attn, OMNIMEM_ERR_INVALID_ARG, "pages: k and v overlap");
  return OMNIMEM_OK;
}
bool on(const Store& x, const Span& a) { return overlap(x.k, a) || overlap(x.v, a); }

const char* kTable = "table must be given, 4-byte aligned";
// The table's entries for rows before `rows`, as an array of bytes.
Span entries(const Store& x, const int32_t* table, int64_t rows) {
  const int64_t bytes = ((rows - 1) >> x.pool.shift) * 4 + 4;
  return {reinterpret_cast<uintptr_t>(table), 1, 1, 0, 0, bytes};
}

}  // namespace

extern "C" {

omnimem_status omnimem_rotate_pages(omnimem_attn* attn, const omnimem_rope* rope, const omnimem_pages* pages,
                                    const omnimem_paged_projection* seqs, int32_t n, hipStream_t stream) {
  omnimem_status st = begin(attn, seqs, n);
  if (st != OMNIMEM_OK) return st;
  const int Hq = attn->cfg.n_q_heads, H = attn->cfg.n_kv_heads;
  PagedRotateArgs<kPagedRotatesPerLaunch> a;
  Store store;
  if ((st = take_rope(attn, rope, a)) != OMNIMEM_OK || (st = take_pages(attn, pages, store)) != OMNIMEM_OK) return st;
  a.pool = store.pool;
  a.n_axes = rope->n_axes;
  for (int i = 0; i < n; ++i) {
    const omnimem_paged_projection& s = seqs[i];
    if (s.n_rows < 0 || s.n_rows > kMaxRows || s.first_row < 0 || s.first_row > kMaxRows - s.n_rows)
      return bad(attn, i, "n_rows or first_row out of range");
    if (s.n_rows == 0) continue;
    if (!readable(attn, s.q, Hq, s.n_rows, s.q_head_stride, s.q_row_stride) ||
        !readable(attn, s.k, H, s.n_rows, s.kv_head_stride, s.kv_row_stride) ||
        !readable(attn, s.v, H, s.n_rows, s.kv_head_stride, s.kv_row_stride))
      return fail(attn, OMNIMEM_ERR_INVALID_ARG, "sequence %d: q, k and v %s", i, kStride);
    if (!s.pos || !aligned(s.pos, 4) || s.pos_stride < 0 || s.pos_stride >= kMaxSpan / 16)
      return bad(attn, i, "pos must be given, 4-byte aligned, its stride >= 0 and below 2^42");
    if (!writable(attn, s.q_out, Hq, s.n_rows, s.q_out_head_stride, s.q_out_row_stride))
      return fail(attn, OMNIMEM_ERR_INVALID_ARG, "sequence %d: q_out %s, no two rows on one place", i, kStride);
    if (!s.table || !aligned(s.table, 4)) return bad(attn, i, kTable);
    const Span q = span(attn, s.q, Hq, s.n_rows, s.q_head_stride, s.q_row_stride);
    const Span k = span(attn, s.k, H, s.n_rows, s.kv_head_stride, s.kv_row_stride);
    const Span v = span(attn, s.v, H, s.n_rows, s.kv_head_stride, s.kv_row_stride);
    const Span o = span(attn, s.q_out, Hq, s.n_rows, s.q_out_head_stride, s.q_out_row_stride);
    const Span table = entries(store, s.table, s.first_row + s.n_rows);
    if (on(store, q) || on(store, k) || on(store, v) || on(store, o) || on(store, table))
      return bad(attn, i, "q, k, v, q_out or the table overlaps the pages");
    if ((!same(o, q) && overlap(o, q)) || overlap(o, k) || overlap(o, v) || overlap(o, table))
      return bad(attn, i, "q_out overlaps an input that it is not");
    if (beside_rows(attn, *rope, s, [&](const Span& x) { return overlap(o, x) || on(store, x); }))
      return bad(attn, i, "q_out or the pages overlap pos or a norm's weights");
  }
  OnDevice dev(attn->device);
  hipError_t e = dev.err;
  const int64_t per = 16 / (int64_t)elt(attn);
  const auto units = [per](int64_t stride) { return (uint32_t)(stride / per); };
  for (int i0 = 0; i0 < n && e == hipSuccess;) {
    int m = 0;
    for (; i0 < n && m < kPagedRotatesPerLaunch; ++i0) {
      const omnimem_paged_projection& s = seqs[i0];
      if (s.n_rows == 0) continue;
      a.seq[m++] = {s.q, s.k, s.v, s.pos, s.q_out, s.table, s.pos_stride, units(s.q_head_stride), units(s.q_row_stride),
                    units(s.kv_head_stride), units(s.kv_row_stride), units(s.q_out_head_stride), units(s.q_out_row_stride),
                    (int32_t)s.first_row, (int32_t)s.n_rows};
    }
    if (m) e = launch_rotate_pages(attn->dm, a, m, stream);
  }
  return done(attn, e, "omnimem_rotate_pages");
}

omnimem_status omnimem_attend_pages(omnimem_attn* attn, const omnimem_pages* pages, const omnimem_paged_query* seqs,
                                    int32_t n, int64_t window, int64_t sinks, hipStream_t stream) {
  omnimem_status st = begin(attn, seqs, n);
  if (st != OMNIMEM_OK) return st;
  const omnimem_attn_config& c = attn->cfg;
  const int Hq = c.n_q_heads, H = c.n_kv_heads;
  Store store;
  if ((st = take_pages(attn, pages, store)) != OMNIMEM_OK) return st;
  if (window < 0 || sinks < 0) return fail(attn, OMNIMEM_ERR_INVALID_ARG, "window and sinks must be >= 0");
  for (int i = 0; i < n; ++i) {
    const omnimem_paged_query& s = seqs[i];
    if (s.n_queries < 0 || s.n_queries > kMaxRows / attn->dm.group || s.memory_rows < 0 || s.memory_rows > kMaxRows ||
        s.n_tail < 0 || s.n_tail > kMaxRows)
      return bad(attn, i, "n_queries, memory_rows or n_tail out of range");
    if (s.n_queries == 0) continue;
    if (!std::isfinite(log2_scale(s, c.head_dim))) return bad(attn, i, "sm_scale times log2(e) is not finite");
    if (!readable(attn, s.q, Hq, s.n_queries, s.q_head_stride, s.q_row_stride))
      return fail(attn, OMNIMEM_ERR_INVALID_ARG, "sequence %d: q %s", i, kStride);
    if (s.n_tail > 0 && (!s.table || !aligned(s.table, 4))) return bad(attn, i, kTable);
    if (s.tree && (!aligned(s.tree, 8) || s.n_queries > kMaxDrafts || s.n_tail < s.n_queries))
      return bad(attn, i, "tree must be 8-byte aligned, its drafts at most 64 and tail rows");
    const int64_t bytes = omnimem_memory_bytes(c.head_dim, s.memory_rows);
    if (s.memory_rows > 0 && (!s.memory || !aligned(s.memory, 16) || s.memory_head_stride % 16 || s.memory_head_stride < 0 ||
                              s.memory_head_stride / 16 > UINT32_MAX || (H > 1 && s.memory_head_stride < bytes)))
      return bad(attn, i, "memory must be given, 16-byte aligned, its head stride a multiple of 16 and at least a head's bytes");
    if (!writable(attn, s.out, Hq, s.n_queries, s.out_head_stride, s.out_row_stride))
      return fail(attn, OMNIMEM_ERR_INVALID_ARG, "sequence %d: out %s, no two rows on one place", i, kStride);
    if (s.lse && (!aligned(s.lse, 4) || s.lse_head_stride < (Hq > 1 ? s.n_queries : 0) || s.lse_head_stride > UINT32_MAX))
      return bad(attn, i, "lse must be 4-byte aligned, its head stride at least n_queries and below 2^32");
    const Span q = span(attn, s.q, Hq, s.n_queries, s.q_head_stride, s.q_row_stride);
    const Span o = span(attn, s.out, Hq, s.n_queries, s.out_head_stride, s.out_row_stride);
    const Span lse = {reinterpret_cast<uintptr_t>(s.lse), Hq, 1, s.lse_head_stride * 4, s.n_queries * 4, s.n_queries * 4};
    const auto written = [&](const Span& x) { return overlap(o, x) || (s.lse && overlap(lse, x)); };
    if (written(q) || (s.lse && overlap(o, lse)) || written(store.k) || written(store.v) ||
        (s.n_tail > 0 && written(entries(store, s.table, s.n_tail))) ||
        (s.tree && written({reinterpret_cast<uintptr_t>(s.tree), 1, 1, 0, 0, s.n_queries * 8})) ||
        (s.memory_rows > 0 && written({reinterpret_cast<uintptr_t>(s.memory), H, 1, s.memory_head_stride, bytes, bytes})))
      return bad(attn, i, "out or lse overlaps the other, q, the pages, the memory, the table or the tree");
  }
  OnDevice dev(attn->device);
  hipError_t e = dev.err;
  const int64_t per = 16 / (int64_t)elt(attn);
  const auto units = [per](int64_t stride) { return (uint32_t)(stride / per); };
  for (int i0 = 0; i0 < n && e == hipSuccess;) {
    PagedArgs<kQueriesPerLaunch> a;
    a.pool = store.pool;
    a.window = (int32_t)(window == 0 ? kMaxRows : std::min(window, kMaxRows));   // (a tail has no more rows)
    a.sinks = (int32_t)std::min(sinks, kMaxRows);
    int m = 0;
    for (; i0 < n && m < kQueriesPerLaunch; ++i0) {
      const omnimem_paged_query& s = seqs[i0];
      if (s.n_queries == 0) continue;
      QuerySeq& x = a.seq[m++];
      x.q = s.q; x.mem = static_cast<const char*>(s.memory); x.k = s.table; x.v = s.tree; x.out = s.out; x.lse = s.lse;
      x.q_hs = units(s.q_head_stride); x.q_rs = units(s.q_row_stride);
      x.kv_hs = x.kv_rs = 0;
      x.out_hs = units(s.out_head_stride); x.out_rs = units(s.out_row_stride);
      x.mem_hs = (uint32_t)(s.memory_head_stride / 16); x.lse_hs = (uint32_t)s.lse_head_stride;
      x.scale_log2 = log2_scale(s, c.head_dim);
      x.nq = (int32_t)s.n_queries; x.nm = (int32_t)s.memory_rows; x.nt = (int32_t)s.n_tail;
    }
    if (m) e = launch_attend_pages(attn->dm, a, m, attn->compute_units, attn->workspace, stream);
  }
  return done(attn, e, "omnimem_attend_pages");
}

omnimem_status omnimem_keep_pages(omnimem_attn* attn, const omnimem_pages* layers, int32_t n_layers,
                                  const omnimem_path* seqs, int32_t n, hipStream_t stream) {
  omnimem_status st = begin(attn, seqs, n);
  if (st != OMNIMEM_OK) return st;
  if (n_layers < 0 || (n_layers > 0 && !layers)) return fail(attn, OMNIMEM_ERR_INVALID_ARG, "null layers, or n_layers < 0");
  Store store;
  // of the layers so far; one that is outside of both (layers' stores one behind the other) is not compared with each
  Range keys, values;
  for (int l = 0; l < n_layers; ++l) {
    if ((st = take_pages(attn, layers + l, store)) != OMNIMEM_OK) return st;
    const omnimem_pages &p = layers[l], &f = layers[0];
    if (p.page_stride != f.page_stride || p.head_stride != f.head_stride || p.row_stride != f.row_stride ||
        p.n_pages != f.n_pages || p.page_rows != f.page_rows)
      return fail(attn, OMNIMEM_ERR_INVALID_ARG, "layer %d: its pages differ from the first layer's", l);
    const bool outside = keys.apart(p.k, store.extent) && values.apart(p.k, store.extent) &&
                         keys.apart(p.v, store.extent) && values.apart(p.v, store.extent);
    keys.add(p.k, store.extent);
    values.add(p.v, store.extent);
    for (int j = 0; j < l && !outside; ++j)
      if (meet(store, apart_by(p.k, layers[j].k)) || meet(store, apart_by(p.v, layers[j].v)) ||
          meet(store, apart_by(p.k, layers[j].v)) || meet(store, apart_by(p.v, layers[j].k)))
        return fail(attn, OMNIMEM_ERR_INVALID_ARG, "layer %d: its pages overlap layer %d's", l, j);
  }
  for (int i = 0; i < n; ++i) {
    const omnimem_path& s = seqs[i];
    if (s.n_kept < 0 || s.n_kept > kMaxDrafts || s.first_row < 0 || s.first_row > kMaxRows - kMaxDrafts)
      return bad(attn, i, "n_kept or first_row out of range");
    if (s.n_kept == 0) continue;
    if (!s.table || !aligned(s.table, 4)) return bad(attn, i, kTable);
    if (!s.path) return bad(attn, i, "null path");
    for (int j = 0; j < s.n_kept; ++j)
      if (s.path[j] >= kMaxDrafts || (j > 0 && s.path[j] <= s.path[j - 1])) return bad(attn, i, "path must ascend, below 64");
    for (int l = 0; l < n_layers; ++l) {
      store.k.base = reinterpret_cast<uintptr_t>(layers[l].k);
      store.v.base = reinterpret_cast<uintptr_t>(layers[l].v);
      if (on(store, entries(store, s.table, s.first_row + s.path[s.n_kept - 1] + 1))) return bad(attn, i, "the table overlaps the pages");
    }
  }
  OnDevice dev(attn->device);
  hipError_t e = dev.err;
  for (int i0 = 0; i0 < n && n_layers > 0 && e == hipSuccess;) {
    KeepArgs a;
    a.pool = store.pool;
    int m = 0;
    for (; i0 < n && m < kKeptPerLaunch; ++i0) {
      const omnimem_path& s = seqs[i0];
      int skip = 0;
      while (skip < s.n_kept && s.path[skip] == skip) ++skip;        // (these are in their place)
      if (skip == s.n_kept) continue;
      KeptSeq& x = a.seq[m++];
      x = {s.table, (int32_t)s.first_row, (uint8_t)skip, (uint8_t)s.n_kept, {}};
      std::copy(s.path, s.path + s.n_kept, x.path);
    }
    for (int l0 = 0; l0 < n_layers && m && e == hipSuccess; l0 += kStoresPerLaunch) {
      const int stores = std::min(kStoresPerLaunch, n_layers - l0);
      for (int l = 0; l < stores; ++l) {
        a.k[l] = static_cast<char*>(layers[l0 + l].k);
        a.v[l] = static_cast<char*>(layers[l0 + l].v);
      }
      e = launch_keep(attn->dm, a, m, stores, stream);
    }
  }
  return done(attn, e, "omnimem_keep_pages");
}

}  // extern "C"
