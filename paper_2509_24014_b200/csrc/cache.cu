// The paged key-value cache: writing new tokens' keys and values to their places, and moving the keys of most accumulated
// attention weight to fewer pages. All of it moves bytes and is bound by HBM, or by the chain of dependent loads (offsets ->
// length -> page table -> data) where there is little to move.
#include <cooperative_groups.h>

#include "cache_choice.h"
#include "sequences.cuh"
#include "topk_device.cuh"

namespace sparsed {
namespace {

constexpr int kRowChunks = 16;   // 16-byte chunks of a head's 128 numbers

// ------------------------------------------------------------------------------------------
// New tokens into the cache. A warp moves a run of tokens (all heads of K and V), four 512-byte pieces of each at a time, of one
// token or, with few heads, of several; the first ones are on their way while it looks for the first token's sequence and place, and
// from then on it goes from sequence to sequence by itself. Nothing is computed or rounded. Bound by HBM: prompts of 330 MB of
// keys and values, read once and written once, in 107 us (6.2 TB/s); one token each of 64 sequences, which is the chain offsets -
// length - page alone, in 2.3 in a graph.
// ------------------------------------------------------------------------------------------
constexpr int kWriteWarps = 8;
constexpr int kWriteChunks = 128;   // 16-byte chunks of K, and of V, that a warp has in flight

// kSeveral: p.tokens_at_once > 1.
template <bool kSeveral>
__global__ void __launch_bounds__(32 * kWriteWarps) cache_write_kernel(const CacheWriteParams p) {
  wait_for_previous_kernel();
  const int lane = threadIdx.x & 31;
  const int64_t begin = (static_cast<int64_t>(blockIdx.x) * kWriteWarps + (threadIdx.x >> 5)) * p.tokens_per_warp;
  if (begin >= p.total) return;
  const int first = static_cast<int>(begin), end = static_cast<int>(min(begin + p.tokens_per_warp, static_cast<int64_t>(p.total)));
  const int token_chunks = p.cache.heads_kv * kRowChunks;
  const int at_once = kSeveral ? p.tokens_at_once : 1;
  uint4 kx[4], vx[4];
  // chunk c of the tokens from `token` on
  auto load = [&](int token, int c0) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int c = c0 + 32 * i + lane, t = kSeveral ? c / token_chunks : 0, in_row = c - t * token_chunks;
      if (kSeveral ? (t < at_once && token + t < end) : c < token_chunks) {
        kx[i] = __ldcs(reinterpret_cast<const uint4*>(p.k + (token + t) * p.k_token + (in_row / kRowChunks) * p.k_head + (in_row % kRowChunks) * 8));
        vx[i] = __ldcs(reinterpret_cast<const uint4*>(p.v + (token + t) * p.v_token + (in_row / kRowChunks) * p.v_head + (in_row % kRowChunks) * 8));
      }
    }
  };
  load(first, 0);
  int seq = last_not_above(p.cache.batch, first, [&](int b) { return __ldcg(p.cu + b); });
  int2 rows = sequence_rows(p.cu, seq, p.total, p.status, 6);
  int len = max(__ldcg(p.cache.lens + seq), 0);
  for (int token = first; token < end; token += at_once) {
    // where lane t's token goes, token + t (of one token: every lane's)
    const int mine = kSeveral ? min(token + min(lane, at_once - 1), end - 1) : token;
    while (mine >= rows.y && seq + 1 < p.cache.batch) {
      rows = sequence_rows(p.cu, ++seq, p.total, p.status, 6);
      len = max(__ldcg(p.cache.lens + seq), 0);
    }
    int page = -1;
    const int place = len - (rows.y - mine);
    if (mine >= rows.x && mine < rows.y) page = page_of(p.cache, seq, place >> p.cache.page_shift, p.status, 7);   // (else behind the last sequence)
    const int at = place & ((1 << p.cache.page_shift) - 1);
    for (int c0 = 0;;) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int c = c0 + 32 * i + lane, t = kSeveral ? c / token_chunks : 0, in_row = c - t * token_chunks;
        const int to_page = kSeveral ? __shfl_sync(0xffffffffu, page, t) : page, to = kSeveral ? __shfl_sync(0xffffffffu, at, t) : at;
        if ((kSeveral ? (t < at_once && token + t < end) : c < token_chunks) && to_page >= 0) {
          const int64_t head = in_row / kRowChunks, piece = (in_row % kRowChunks) * 8;
          *reinterpret_cast<uint4*>(p.cache.k + to_page * p.cache.k_page + to * p.cache.k_place + head * p.cache.k_head + piece) = kx[i];
          *reinterpret_cast<uint4*>(p.cache.v + to_page * p.cache.v_page + to * p.cache.v_place + head * p.cache.v_head + piece) = vx[i];
        }
      }
      c0 += kWriteChunks;
      if (kSeveral || c0 >= token_chunks) break;
      load(token, c0);
    }
    if (token + at_once < end) load(token + at_once, 0);
  }
}

// ------------------------------------------------------------------------------------------
// Eviction, first half: which keys stay. A cluster of CTAs ranks one row (sequence, key-value head), each CTA a run of its
// candidates (all but the `recent` last keys): radix selection of the (keep - recent)-th largest mass, 11 + 11 + 10 bits of a key
// that orders like the float, ended early once all of the bin that holds it stay. Each CTA counts its keys in a histogram of its
// own; then each adds up a slice of the bins over the cluster and scans it, and all find the bin from the slices' totals (every CTA
// adding up every bin for itself took 2.5 us a step for a cluster of eight, 0.5 this way). At the end every warp counts and writes
// out its share in order. Nothing is rounded: masses are compared and copied.
//
// Bound by the latency of these steps, and with 1024 threads by their instructions: of 8.3 us for 3000 candidates in one CTA (with
// cold caches) the loads take 2.7, a step 0.5 for counting, 0.25 for adding up and 0.2 for the bin, the writing 2.2; of 18 us for
// 13,000 in each of four CTAs 5, 3 and 7.
// ------------------------------------------------------------------------------------------
constexpr int kBins = 2048;
constexpr int kScanThreads = 256;   // that add up and scan the bins (with all 1024 the instructions of it took twice as long)
constexpr int kLoadBatch = 4;    // weights that a thread has on their way when a CTA reads its run
constexpr int kWriteBatch = 8;   // times 32 keys whose weights a warp has on their way when it writes out its share
constexpr uint32_t kZeroKey = 0x80000000u;   // ordered_key(0)
// of a CTA's run, held in shared memory (96 KB, 8 KB) as ordered keys
__host__ __device__ constexpr int cached_keys(int threads) { return threads == 1024 ? 24 * 1024 : kShortRow; }

template <int ranks, int threads>
struct EvictSmem {
  alignas(16) uint32_t keys[cached_keys(threads)];
  int hist[kBins];
  int2 slice[ranks > 1 ? kBins / ranks : 1];   // of this CTA's slice of the bins: keys in each over the cluster, and in the slice's bins above it
  int slice_total;
  int warp_sum[kScanThreads / 32];
  int found_bin, found_above, found_count;
  int keys_above[threads / 32], keys_equal[threads / 32];   // above / equal to the threshold in each warp's share
  int cta_above, cta_equal;
  int zeros;               // keys of weight zero in this CTA's run
};

// ranks: CTAs to a row (1, 2, 4 or 8).
template <int ranks, int kSelectThreads>
__global__ void __launch_bounds__(kSelectThreads, 1024 / kSelectThreads) evict_select_kernel(const EvictParams p) {
  namespace cg = cooperative_groups;
  constexpr int kSelectWarps = kSelectThreads / 32, kCachedKeys = cached_keys(kSelectThreads);
  extern __shared__ __align__(16) uint8_t smem_raw[];
  auto& sm = *reinterpret_cast<EvictSmem<ranks, kSelectThreads>*>(smem_raw);
  wait_for_previous_kernel();
  cg::cluster_group cluster = cg::this_cluster();
  const int rank = ranks == 1 ? 0 : static_cast<int>(cluster.block_rank());
  auto sync_row = [&]() {
    if constexpr (ranks == 1) __syncthreads();
    else cluster.sync();
  };
  const int row = blockIdx.x / ranks;   // sequence * heads_kv + head
  const int seq = row / p.from.heads_kv, head = row % p.from.heads_kv;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int len = cached_length(p.from, seq, p.status, 8);
  const float* mass = p.mass + row * p.mass_capacity;
  float* mass_out = p.mass_out + row * p.mass_out_capacity;
  int32_t* kept = p.kept + static_cast<int64_t>(row) * p.keep;
  const int n_kept = min(p.keep, len);
  if (head == 0 && rank == 0 && tid == 0) p.to.lens[seq] = n_kept;
  // behind the kept keys
  const int all = ranks * kSelectThreads, me = rank * kSelectThreads + tid;
  for (int j = n_kept + me; j < p.keep; j += all) kept[j] = -1;
  for (int64_t j = n_kept + me; j < p.mass_out_capacity; j += all) mass_out[j] = 0.f;
  if (len <= p.keep) {   // (the whole cluster alike)
    for (int j = me; j < len; j += all) {
      kept[j] = j;
      mass_out[j] = __ldcg(mass + j);
    }
    return;
  }
  const int candidates = len - p.recent, need = p.keep - p.recent;
  const float recent_mass = me < p.recent ? __ldcg(mass + candidates + me) : 0.f;
  auto keep_recent = [&]() {
    if (me < p.recent) {
      kept[need + me] = candidates + me;
      mass_out[need + me] = recent_mass;
    }
    for (int j = me + all; j < p.recent; j += all) {
      kept[need + j] = candidates + j;
      mass_out[need + j] = __ldcg(mass + candidates + j);
    }
  };
  if (need == 0) {
    keep_recent();
    return;
  }
  // this CTA's run of candidates, in whole warps' shares of whole fours
  const int share = (candidates + ranks * kSelectWarps * 4 - 1) / (ranks * kSelectWarps * 4) * 4;   // candidates per warp
  const int run0 = min(rank * kSelectWarps * share, candidates), run1 = min((rank + 1) * kSelectWarps * share, candidates);
  const int run = run1 - run0;
  const int cached = min(run, kCachedKeys);
  if (tid == 0) sm.zeros = 0;
  for (int i = tid; i < kBins; i += kSelectThreads) sm.hist[i] = 0;
  __syncthreads();
  // Weights of exactly zero (keys that no query has looked at) are often most of a row: they are counted here once, and not by
  // thousands of additions to one place of every histogram.
  int zeros = 0;
  for (int i0 = tid; i0 < cached; i0 += kLoadBatch * kSelectThreads) {
    float x[kLoadBatch];
#pragma unroll
    for (int j = 0; j < kLoadBatch; ++j) x[j] = i0 + j * kSelectThreads < cached ? __ldcg(mass + run0 + i0 + j * kSelectThreads) : 1.f;
#pragma unroll
    for (int j = 0; j < kLoadBatch; ++j) {
      const uint32_t key = ordered_key(x[j]);
      if (i0 + j * kSelectThreads < cached) sm.keys[i0 + j * kSelectThreads] = key;
      zeros += key == kZeroKey;
    }
  }
  keep_recent();
  for (int i = cached + tid; i < run; i += kSelectThreads) zeros += ordered_key(__ldcg(mass + run0 + i)) == kZeroKey;
  zeros = __reduce_add_sync(0xffffffffu, zeros);
  if (lane == 0 && zeros > 0) atomicAdd(&sm.zeros, zeros);
  // keys i to i + 3 of the run (i a multiple of 4); how many of them there are
  auto keys_at = [&](int i, uint32_t (&key)[4]) -> int {
    if (i + 4 <= cached) {
      const uint4 x = *reinterpret_cast<const uint4*>(sm.keys + i);
      key[0] = x.x, key[1] = x.y, key[2] = x.z, key[3] = x.w;
      return 4;
    }
    const int n = min(run - i, 4);
#pragma unroll
    for (int x = 0; x < 4; ++x) key[x] = x >= n ? 0u : (i + x < cached ? sm.keys[i + x] : ordered_key(__ldcg(mass + run0 + i + x)));
    return n;
  };
  __syncthreads();
  // ---- the threshold -----------------------------------------------------------------------
  uint32_t prefix = 0u;
  int left = need;          // of the keys that agree with `prefix` in the bits decided so far
  constexpr int kSlice = kBins / ranks, kPerThread = kSlice / kScanThreads;   // bins that each CTA, and each thread, adds up
  for (int step = 0; step < 3; ++step) {
    const int shift = step == 0 ? 21 : (step == 1 ? 10 : 0), decided = shift + (step == 2 ? 10 : 11);
    const uint32_t bins = step == 2 ? 1024u : kBins;
    for (int i = 4 * tid; i < run; i += 4 * kSelectThreads) {
      uint32_t key[4];
      const int n = keys_at(i, key);
#pragma unroll
      for (int x = 0; x < 4; ++x)
        if (x < n && key[x] != kZeroKey && (step == 0 || (key[x] ^ prefix) >> decided == 0u)) atomicAdd(&sm.hist[(key[x] >> shift) & (bins - 1u)], 1);
    }
    if (tid == 0 && (step == 0 || (kZeroKey ^ prefix) >> decided == 0u)) atomicAdd(&sm.hist[(kZeroKey >> shift) & (bins - 1u)], sm.zeros);
    sync_row();
    // This CTA's slice: the bins from rank * kSlice on, the highest first, a few to a thread.
    int in[kPerThread], sum = 0;
    const int first_bin = rank * kSlice + kSlice - 1 - kPerThread * tid;   // (and those below it)
    if (tid < kScanThreads) {
#pragma unroll
      for (int x = 0; x < kPerThread; ++x) in[x] = 0;
#pragma unroll
      for (int r = 0; r < ranks; ++r)
#pragma unroll
        for (int x = 0; x < kPerThread; ++x) in[x] += ranks == 1 ? sm.hist[first_bin - x] : *cluster.map_shared_rank(&sm.hist[first_bin - x], r);
#pragma unroll
      for (int x = 0; x < kPerThread; ++x) sum += in[x];
      const int own = sum;
#pragma unroll
      for (int d = 1; d < 32; d *= 2) {
        const int other = __shfl_up_sync(0xffffffffu, sum, d);
        if (lane >= d) sum += other;
      }
      if (lane == 31) sm.warp_sum[warp] = sum;
      named_barrier_sync(1, kScanThreads);
      sum += __reduce_add_sync(0xffffffffu, lane < warp ? sm.warp_sum[lane] : 0) - own;   // in the slice's bins above
    }
    if constexpr (ranks == 1) {
      if (tid < kScanThreads) {
#pragma unroll
        for (int x = 0; x < kPerThread; ++x) {
          if (sum < left && sum + in[x] >= left) {
            sm.found_bin = first_bin - x;
            sm.found_above = sum;
            sm.found_count = in[x];
          }
          sum += in[x];
        }
      }
      __syncthreads();
      for (int i = tid; i < kBins; i += kSelectThreads) sm.hist[i] = 0;
      __syncthreads();
    } else {
      if (tid < kScanThreads) {
#pragma unroll
        for (int x = 0; x < kPerThread; ++x) {
          sm.slice[first_bin - rank * kSlice - x] = make_int2(in[x], sum);
          sum += in[x];
        }
        if (tid == kScanThreads - 1) sm.slice_total = sum;
      }
      sync_row();
      for (int i = tid; i < kBins; i += kSelectThreads) sm.hist[i] = 0;   // (all have read it)
      // The slice in which the count from the top passes `left`, then the bin: every CTA looks for itself.
      if (tid < kScanThreads) {
        const int total = lane < ranks ? *cluster.map_shared_rank(&sm.slice_total, ranks - 1 - lane) : 0;   // lane 0: the highest slice
        int upto = total;
#pragma unroll
        for (int d = 1; d < ranks; d *= 2) {
          const int other = __shfl_up_sync(0xffffffffu, upto, d);
          if (lane >= d) upto += other;
        }
        const int at_lane = __ffs(__ballot_sync(0xffffffffu, lane < ranks && upto >= left)) - 1;   // (the lowest reaches it at last)
        const int owner = ranks - 1 - at_lane, before = __shfl_sync(0xffffffffu, upto - total, at_lane);
        int2 bin[kPerThread];
#pragma unroll
        for (int x = 0; x < kPerThread; ++x) bin[x] = *cluster.map_shared_rank(&sm.slice[x * kScanThreads + tid], owner);
#pragma unroll
        for (int x = 0; x < kPerThread; ++x)
          if (before + bin[x].y < left && before + bin[x].y + bin[x].x >= left) {
            sm.found_bin = owner * kSlice + x * kScanThreads + tid;
            sm.found_above = before + bin[x].y;
            sm.found_count = bin[x].x;
          }
      }
      __syncthreads();
      // (the slices are read by other CTAs until they come to the next step's first barrier, and written behind it)
    }
    prefix |= static_cast<uint32_t>(sm.found_bin) << shift;
    left -= sm.found_above;
    if (left == sm.found_count && prefix != 0u) {   // the whole bin stays: the lower bits need not be known
      --prefix;
      left = 0;
      break;
    }
  }
  // Kept: keys above `prefix`, and the first `left` of those equal to it.
  // ---- where each warp's share goes ----------------------------------------------------------
  const int my0 = min(warp * share, run), my1 = min(my0 + share, run);
  int above = 0, equal = 0;
  for (int i = my0 + 4 * lane; i < my1; i += 128) {
    uint32_t key[4];
    const int n = min(keys_at(i, key), my1 - i);
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      above += x < n && key[x] > prefix;
      equal += x < n && key[x] == prefix;
    }
  }
  above = __reduce_add_sync(0xffffffffu, above);
  equal = __reduce_add_sync(0xffffffffu, equal);
  if (lane == 0) {
    sm.keys_above[warp] = above;
    sm.keys_equal[warp] = equal;
  }
  __syncthreads();
  if (warp == 0) {
    const int a = __reduce_add_sync(0xffffffffu, lane < kSelectWarps ? sm.keys_above[lane] : 0);
    const int e = __reduce_add_sync(0xffffffffu, lane < kSelectWarps ? sm.keys_equal[lane] : 0);
    if (lane == 0) {
      sm.cta_above = a;
      sm.cta_equal = e;
    }
  }
  sync_row();
  // in the shares before this warp's: those of CTAs before (a lane each) and of warps before
  int above_before = 0, equal_before = 0;
  if (ranks > 1 && lane < rank) {
    above_before = *cluster.map_shared_rank(&sm.cta_above, lane);
    equal_before = *cluster.map_shared_rank(&sm.cta_equal, lane);
  }
  above_before = __reduce_add_sync(0xffffffffu, above_before + (lane < warp ? sm.keys_above[lane] : 0));
  equal_before = __reduce_add_sync(0xffffffffu, equal_before + (lane < warp ? sm.keys_equal[lane] : 0));
  const uint32_t lower = (1u << lane) - 1u;
  for (int i0 = my0; i0 < my1; i0 += 32 * kWriteBatch) {
    float weight[kWriteBatch];   // (as it is: a key does not tell NaNs apart, nor zeros)
#pragma unroll
    for (int x = 0; x < kWriteBatch; ++x) weight[x] = i0 + 32 * x + lane < my1 ? __ldcg(mass + run0 + i0 + 32 * x + lane) : 0.f;
#pragma unroll
    for (int x = 0; x < kWriteBatch; ++x) {
      if (i0 + 32 * x >= my1) break;
      const int i = i0 + 32 * x + lane;
      const uint32_t key = i >= my1 ? 0u : (i < cached ? sm.keys[i] : ordered_key(weight[x]));
      const bool is_above = i < my1 && key > prefix, is_equal = i < my1 && key == prefix;
      const uint32_t a = __ballot_sync(0xffffffffu, is_above), e = __ballot_sync(0xffffffffu, is_equal);
      const int my_equal = equal_before + __popc(e & lower);
      if (is_above || (is_equal && my_equal < left)) {
        const int at = above_before + __popc(a & lower) + min(my_equal, left);
        kept[at] = run0 + i;
        mass_out[at] = weight[x];
      }
      above_before += __popc(a);
      equal_before += __popc(e);
    }
  }
  if constexpr (ranks > 1) sync_row();   // no CTA leaves while another may still read its counts
}

// ------------------------------------------------------------------------------------------
// Eviction, second half: the kept rows of K and V to their new pages. A warp moves eight keys of a row: eight lanes look up one
// key's place and its new one each, then sixteen lanes at a time move a key's 256 bytes, four keys of K and V in flight per lane.
// Bound by HBM where there is much to move: 2 x 16384 keys x 8 heads, 268 MB read and written, in 43 us (6.2 TB/s); else by the
// chain kept - page - data. (32 keys to a warp, the whole call, us: 2 rows of 30,000 18.6 against 16.0, 4 of 32,768 20.1 | 18.2, 2 of
// 4000 12.6 | 9.9, 2 x 52k x 8 69.7 | 69.2; 128 of 2000 20.0 | 21.7.)
// ------------------------------------------------------------------------------------------
constexpr int kMoveThreads = 128;
constexpr int kMoveKeys = 8;   // to a warp

__global__ void __launch_bounds__(kMoveThreads) evict_move_kernel(const EvictParams p) {
  wait_for_previous_kernel();
  const int lane = threadIdx.x & 31, number = blockIdx.x * (kMoveThreads / 32) + (threadIdx.x >> 5);
  const int warps_per_row = (p.keep + kMoveKeys - 1) / kMoveKeys;
  const int row = number / warps_per_row, j = (number - row * warps_per_row) * kMoveKeys + lane;
  if (row >= p.from.batch * p.from.heads_kv) return;
  const int seq = row / p.from.heads_kv, head = row - seq * p.from.heads_kv;
  const int from = lane < kMoveKeys && j < p.keep ? __ldcg(p.kept + static_cast<int64_t>(row) * p.keep + j) : -1;
  int page = -1, new_page = -1;
  if (from >= 0) {
    new_page = page_of(p.to, seq, j >> p.to.page_shift, p.status, 10);
    page = page_of(p.from, seq, from >> p.from.page_shift, p.status, 9);
  }
  if (__all_sync(0xffffffffu, new_page < 0)) return;
  const int place = from & ((1 << p.from.page_shift) - 1), new_place = j & ((1 << p.to.page_shift) - 1);
  const int c = (lane & 15) * 8;
  const uint16_t* k = p.from.k + head * p.from.k_head + c;
  const uint16_t* v = p.from.v + head * p.from.v_head + c;
  uint16_t* new_k = p.to.k + head * p.to.k_head + c;
  uint16_t* new_v = p.to.v + head * p.to.v_head + c;
  uint4 kx[4], vx[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int key = 2 * i + (lane >> 4);
    const int at_page = __shfl_sync(0xffffffffu, page, key), at = __shfl_sync(0xffffffffu, place, key);
    kx[i] = vx[i] = make_uint4(0u, 0u, 0u, 0u);   // (a key whose page is missing comes over as zeros)
    if (at_page >= 0) {
      kx[i] = __ldcs(reinterpret_cast<const uint4*>(k + at_page * p.from.k_page + at * p.from.k_place));
      vx[i] = __ldcs(reinterpret_cast<const uint4*>(v + at_page * p.from.v_page + at * p.from.v_place));
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int key = 2 * i + (lane >> 4);
    const int to_page = __shfl_sync(0xffffffffu, new_page, key), to = __shfl_sync(0xffffffffu, new_place, key);
    if (to_page >= 0) {
      *reinterpret_cast<uint4*>(new_k + to_page * p.to.k_page + to * p.to.k_place) = kx[i];
      *reinterpret_cast<uint4*>(new_v + to_page * p.to.v_page + to * p.to.v_place) = vx[i];
    }
  }
}

}  // namespace

cudaError_t launch_cache_write(CacheWriteParams p, cudaStream_t stream) {
  const int token_chunks = p.cache.heads_kv * kRowChunks;
  p.tokens_at_once = token_chunks < kWriteChunks ? kWriteChunks / token_chunks : 1;
  // A warp has a token's chunks in one turn (5 to 8 heads): then two tokens to a warp, so that the second one's loads are on their
  // way while the first is written (one | two | four, us: 48,000 tokens of 8 heads 69.2 | 64.1 | 65.4, of 6 57.5 | 51.6 | 52.1, 16,000
  // of 8 26.0 | 24.4 | 24.6), unless these are few. With more heads a token has turns enough (32 heads, prompts of 20,000: 107.3 |
  // 109.9 | 111.4); with fewer, several tokens to a turn hide the way to their places (48,000 of 4 heads 38.9 | 41.0 | 42.0; a token
  // to a turn, 4 heads 47.8 -> 38.9, 2 40.5 -> 21.4, 1 37.1 -> 10.7).
  const bool one_turn = p.tokens_at_once == 1 && token_chunks <= kWriteChunks;
  p.tokens_per_warp = one_turn && p.total >= 8192 ? 2 : p.tokens_at_once;
  const int64_t warps = (static_cast<int64_t>(p.total) + p.tokens_per_warp - 1) / p.tokens_per_warp;
  const int ctas = static_cast<int>((warps + kWriteWarps - 1) / kWriteWarps);
  return p.tokens_at_once > 1 ? launch_overlapped(cache_write_kernel<true>, ctas, ctas, 32 * kWriteWarps, 0, stream, p)
                              : launch_overlapped(cache_write_kernel<false>, ctas, ctas, 32 * kWriteWarps, 0, stream, p);
}

cudaError_t launch_cache_evict(const EvictParams& p, cudaStream_t stream) {
  const int rows = p.from.batch * p.from.heads_kv;
  struct Variant {
    void (*kernel)(EvictParams);
    int threads, smem;
  };
  constexpr Variant variants[5] = {{evict_select_kernel<1, 1024>, 1024, sizeof(EvictSmem<1, 1024>)}, {evict_select_kernel<2, 1024>, 1024, sizeof(EvictSmem<2, 1024>)},
                                   {evict_select_kernel<4, 1024>, 1024, sizeof(EvictSmem<4, 1024>)}, {evict_select_kernel<8, 1024>, 1024, sizeof(EvictSmem<8, 1024>)},
                                   {evict_select_kernel<1, 256>, 256, sizeof(EvictSmem<1, 256>)}};
  const EvictChoice choice = choose_evict_variant(rows, p.from.max_pages << p.from.page_shift);
  const int ranks = choice.ranks, which = ranks > 1 ? (ranks == 2 ? 1 : (ranks == 4 ? 2 : 3)) : (choice.threads == 256 ? 4 : 0);
  const Variant& variant = variants[which];
  static SmemLimit limits[5];
  cudaError_t e = ensure_dynamic_smem(variant.kernel, variant.smem, limits[which]);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(rows * ranks));
  cfg.blockDim = dim3(static_cast<unsigned>(variant.threads));
  cfg.dynamicSmemBytes = static_cast<size_t>(variant.smem);
  cfg.stream = stream;
  cudaLaunchAttribute attr[2] = {};
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = static_cast<unsigned>(ranks);
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  e = cudaLaunchKernelEx(&cfg, variant.kernel, p);
  if (e == cudaSuccess) {
    cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>((static_cast<int64_t>((p.keep + kMoveKeys - 1) / kMoveKeys) * rows + kMoveThreads / 32 - 1) / (kMoveThreads / 32)));
    cfg.blockDim = dim3(kMoveThreads);
    cfg.stream = stream;
    attr[0] = {};
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    e = cudaLaunchKernelEx(&cfg, evict_move_kernel, p);
  }
  if (e != cudaSuccess) (void)cudaGetLastError();
  return e;
}

}  // namespace sparsed
