// Device-side helpers for sequences of different lengths: finding a sequence by an offset, and places in a paged cache.
#pragma once

#include "packed_and_paged.h"

namespace sparsed {

// The last index b in [0, n) with value(b) <= key, by a whole warp (32 probes a round), for values that ascend; index 0 if
// there is none. Values that do not ascend give some index in range. All lanes return the same.
template <class Value>
__device__ __forceinline__ int last_not_above(int n, int key, Value value) {
  const int lane = threadIdx.x & 31;
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int step = (hi - lo + 31) / 32;
    const int at = lo + lane * step;
    const bool below = at < hi && value(at) <= key;
    const int found = __popc(__ballot_sync(0xffffffffu, below));
    lo += max(found - 1, 0) * step;
    hi = min(hi, lo + step);
  }
  return lo;
}

__device__ __forceinline__ void record_status(DeviceStatus* status, int code, int where) {
  if (atomicCAS(&status->code, 0, code) == 0) status->where = where;
}

// The first and one past the last row of a sequence, clipped to [0, total].
__device__ __forceinline__ int2 clip_rows(int first, int end, int total, DeviceStatus* status, int where) {
  const int f = min(max(first, 0), total), e = min(max(end, f), total);
  if (f != first || e != end) record_status(status, 6, where);
  return make_int2(f, e);
}
__device__ __forceinline__ int2 sequence_rows(const int32_t* cu, int b, int total, DeviceStatus* status, int where) {
  return clip_rows(__ldcg(cu + b), __ldcg(cu + b + 1), total, status, where);
}

// Page of the cache that holds positions [place << page_shift, ...) of sequence b, or -1 where the table has none (recorded).
__device__ __forceinline__ int page_of(const CacheView& c, int b, int place, DeviceStatus* status, int where) {
  int page = -1;
  if (place >= 0 && place < c.max_pages) page = __ldcg(c.table + b * c.table_stride + place);
  if (page < 0 || page >= c.num_pages) {
    record_status(status, 5, where);
    page = -1;
  }
  return page;
}

// Cached positions of sequence b, clipped to what its row of the table can hold.
__device__ __forceinline__ int cached_length(const CacheView& c, int b, DeviceStatus* status, int where) {
  const int len = max(__ldcg(c.lens + b), 0), room = c.max_pages << c.page_shift;
  if (len > room) record_status(status, 5, where);
  return min(len, room);
}

}  // namespace sparsed
