// Which of a warp's loads are still on their way when the one-token kernel (attention_paged.cu) gives up. A warp has one place
// for K and one for V, each with a barrier whose nth use is phase n & 1; it waits for K of tile n, sends K of the next tile off
// (if that has any for this warp), then does the same for V.
#pragma once

#include <stdint.h>

namespace sparsed {

enum class PagedWait { kNone, kKeys, kValues };   // what ran out

struct PagedLoads {
  bool keys, values;   // on their way
  uint32_t keys_use, values_use;   // which use of the barrier counts them
};

// failed: the wait that ran out, in the warp's tile number `use`; next: whether that is followed by another. A warp that has come
// to the end of its segment has nothing on its way.
#ifdef __CUDACC__
__host__ __device__
#endif
constexpr PagedLoads paged_loads_on_their_way(PagedWait failed, uint32_t use, bool next) {
  return {failed == PagedWait::kKeys || (failed == PagedWait::kValues && next), failed != PagedWait::kNone,
          failed == PagedWait::kKeys ? use : use + 1, use};
}

}  // namespace sparsed
