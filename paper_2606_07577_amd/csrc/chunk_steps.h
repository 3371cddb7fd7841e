// The order in which a unit of the chunk attention works on its LDS stages,
// apart from the work itself, so that it can be run on the host too.
#pragma once

#include <type_traits>

#include <hip/hip_runtime.h>

namespace omnimem {

// K and V of the key tiles k0 .. k1 - 1 (the memory's up to mid, then the
// tail's) through four stages of each; tile t has stage (t - k0) & 3.  The
// opening takes K of tile k0 (its scores), and step t takes K of tile t + 1 and
// V of tile t, and brings K of tile t + 3 and V of tile t + 2: fetch at its
// begin, store (for what goes through registers) at its end.  A barrier, which
// also waits for what this wavefront fetched, follows the first tiles, the
// opening and every second step.  The opening stands for a step before the
// first: K of tile t is taken in step t - 1 and its stage is fetched into in
// step t + 1, so one of the two has to end with a barrier, and after the
// opening step 0 does not.  So a barrier lies between a fetch and the first
// step that takes it, and between the last step that takes a stage and the next
// fetch into it.
//   fetch_k, fetch_v, store_k, store_v (tile, stage)
//   first (stage)                               scores of tile k0
//   step (memory, swapped, tile, K stage, V stage)   scores of the next tile in
//                                               one of two places in turn
//   keep ()                                     scores back to the first place
//   barrier ()
template <typename FetchK, typename FetchV, typename StoreK, typename StoreV, typename First, typename Step, typename Keep,
          typename Barrier>
__host__ __device__ __attribute__((always_inline)) inline void chunk_steps(int k0, int k1, int mid, FetchK fetch_k, FetchV fetch_v,
                                                                           StoreK store_k, StoreV store_v, First first, Step step,
                                                                           Keep keep, Barrier barrier) {
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    if (k0 + i < k1) {
      fetch_k(k0 + i, i);
      if (i < 2) fetch_v(k0 + i, i);
      store_k(k0 + i, i);
      if (i < 2) store_v(k0 + i, i);
    }
  }
  barrier();
  first(0);
  barrier();
  const auto one = [&](auto mem, auto swapped, int t) __attribute__((always_inline)) {
    const int i = t - k0;
    if (t + 3 < k1) fetch_k(t + 3, (i + 3) & 3);
    if (t + 2 < k1) fetch_v(t + 2, (i + 2) & 3);
    step(mem, swapped, t, (i + 1) & 3, i & 3);
    if (t + 3 < k1) store_k(t + 3, (i + 3) & 3);
    if (t + 2 < k1) store_v(t + 2, (i + 2) & 3);
    if (i & 1) barrier();
  };
  const auto steps = [&](auto mem, int t, int end) __attribute__((always_inline)) {   // (two at a time: scores stay where they are)
    for (; t + 1 < end; t += 2) {
      one(mem, std::false_type{}, t);
      one(mem, std::true_type{}, t + 1);
    }
    if (t < end) {
      one(mem, std::false_type{}, t);
      keep();
    }
  };
  steps(std::true_type{}, k0, mid);
  steps(std::false_type{}, mid, k1);
}

}  // namespace omnimem
