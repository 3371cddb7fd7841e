// Attention over a memory and tail rows in the pages of a cache.
#include "attend_kernels.h"

namespace omnimem {

hipError_t prepare_attend_pages(const AttnDims& dm) { return prepare<PagedArgs<kQueriesPerLaunch>>(dm); }

hipError_t launch_attend_pages(const AttnDims& dm, PagedArgs<kQueriesPerLaunch>& a, int n, int compute_units, void* ws, hipStream_t st) {
  a.causal = 1;
  return attend_all(dm, a, n, compute_units, ws, st);
}

}  // namespace omnimem
