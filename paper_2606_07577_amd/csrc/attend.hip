// Attention over a memory and tail rows that lie one after the other.
#include "attend_kernels.h"

namespace omnimem {

hipError_t prepare_attend(const AttnDims& dm) {
  const hipError_t e = prepare<AttendArgs<kQueriesPerLaunch>>(dm);
  return e != hipSuccess ? e : prepare_attend_pages(dm);
}

hipError_t launch_attend(const AttnDims& dm, AttendArgs<kQueriesPerLaunch>& a, int n, int compute_units, void* ws, hipStream_t st) {
  return attend_all(dm, a, n, compute_units, ws, st);
}

}  // namespace omnimem
