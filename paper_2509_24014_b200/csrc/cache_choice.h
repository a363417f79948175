// Which variant of the selection kernel an eviction gets (cache.cu).
#pragma once

namespace sparsed {

constexpr int kMostRanks = 8;    // CTAs to a row
constexpr int kShortRow = 2048;  // the most keys of a row that a CTA of 256 threads takes

struct EvictChoice {
  int ranks;     // CTAs to a row: 1, 2, 4 or 8
  int threads;   // to a CTA: 1024, or 256 (of one CTA to a row)
};

// rows: sequences times key-value heads; room: keys that a row of the table has places for.
inline EvictChoice choose_evict_variant(long long rows, int room) {
  // Several CTAs to a row that is long enough to be shared, as long as they take no more than 64 SMs: a CTA needs an SM for
  // itself and a cluster the SMs of one part of the device, so more would not run at the same time. The whole call, us (this and
  // the figures below with 32 keys to a moving warp, which adds 0.5 to 2): 16 rows of
  // 52k in clusters of 8 (two rounds) 74.1, of 4 69.5, of 2 87.0, one CTA to a row 120; 8 rows of 128k, 8 or 4 49.9, 2 74.5,
  // one 123; 4 rows of 32k, 8 19.9, 4 20.2, 2 21.5. Of short rows a cluster's barriers and remote reads cost more than it gains:
  // 32 rows of up to 4k, one CTA 22.2, two 28.1; 16 rows of 8000, one 17.5, two 19.6, four 19.1; 8 of 16000, two 20.7, four 18.9.
  int ranks = 1;
  while (ranks < kMostRanks && rows * ranks * 2 <= 64 && room / (2 * ranks) >= 2048) ranks *= 2;
  // Short rows get CTAs of 256 threads, four to an SM: the call with 1024 | 256 threads, us, 352 rows of up to 59 keys 22.2 | 14.0,
  // 148 of 1000 23.2 | 20.4, 32 of 1000 12.3 | 11.6, 4 of 1000 10.9 | 10.3, 128 of 2000 22.5 | 19.9; but 32 of 2000 13.3 | 13.7 and
  // 256 of 4000 41.6 | 43.3.
  const bool short_rows = room <= (rows > 64 ? kShortRow : kShortRow / 2);
  return {ranks, short_rows ? 256 : 1024};
}

}  // namespace sparsed
