// Accepted drafts of caches in pages to the rows that they become.
#include "../../include/omnimem.h"
#include "attn.h"

namespace omnimem {
namespace {

constexpr int kRowsAhead = 8;

// A thread to 16 bytes of a head's rows of K or of V, which it moves in the
// path's order, kRowsAhead at a time: row path[i] >= i is written to row i, and
// the rows read later are path[j] > path[i] >= i, so no row is written before
// it is read.  Latency bounds it: table entries, a row, and for each 8 rows more
// the same again (7 rows of 8 sequences in 28 layers, 3.3 MB each way, 5.7 us; 4
// rows of one in 4 layers 4.4).
__global__ __launch_bounds__(256) void keep_rows(KeepArgs a, int chunks, int items) {
  const KeptSeq& s = a.seq[blockIdx.y];
  const int item = blockIdx.x * 256 + threadIdx.x;
  if (item >= items) return;
  const int half = items / 2, part = item % half;
  char* base = (item < half ? a.k : a.v)[blockIdx.z] + part / chunks * a.pool.head + part % chunks * 16;
  for (int i0 = s.skip; i0 < s.n; i0 += kRowsAhead) {
    int64_t from[kRowsAhead], to[kRowsAhead];
    uint4 x[kRowsAhead];
#pragma unroll
    for (int i = 0; i < kRowsAhead; ++i) {
      const int j = min(i0 + i, s.n - 1);
      from[i] = paged_row<true>(a.pool, s.table, s.first + s.path[j]);
      to[i] = paged_row<true>(a.pool, s.table, s.first + j);
    }
#pragma unroll
    for (int i = 0; i < kRowsAhead; ++i) x[i] = from[i] >= 0 ? gload16(base + from[i]) : make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int i = 0; i < kRowsAhead; ++i)
      if (i0 + i < s.n && from[i] >= 0 && to[i] >= 0) *reinterpret_cast<uint4*>(base + to[i]) = x[i];
  }
}

}  // namespace

hipError_t launch_keep(const AttnDims& dm, const KeepArgs& a, int n, int stores, hipStream_t st) {
  const int chunks = dm.d * (dm.dtype == OMNIMEM_BF16 ? 2 : 4) / 16, items = 2 * dm.h_kv * chunks;
  keep_rows<<<dim3((unsigned)((items + 255) / 256), n, stores), 256, 0, st>>>(a, chunks, items);
  return hipGetLastError();
}

}  // namespace omnimem
