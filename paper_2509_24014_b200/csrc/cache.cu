// The paged key-value cache: writing new tokens' keys and values to their places, and moving the keys of most accumulated
// attention weight to fewer pages. All of it moves bytes and is bound by HBM, or by the chain of dependent loads (offsets ->
// length -> page table -> data) where there is little to move.
#include <cooperative_groups.h>

#include "sequences.cuh"
#include "topk_device.cuh"

namespace sparsed {
namespace {

constexpr int kRowChunks = 16;   // 16-byte chunks of a head's 128 numbers

// ------------------------------------------------------------------------------------------
// New tokens into the cache. A warp moves one token (all heads of K and V), four 512-byte pieces of each at a time; the first
// ones are on their way while it looks for the token's sequence and place.
// ------------------------------------------------------------------------------------------
constexpr int kWriteWarps = 8;

__global__ void __launch_bounds__(32 * kWriteWarps) cache_write_kernel(const CacheWriteParams p) {
  wait_for_previous_kernel();
  const int lane = threadIdx.x & 31;
  const int token = blockIdx.x * kWriteWarps + (threadIdx.x >> 5);
  if (token >= p.total) return;
  const int chunks = p.cache.heads_kv * kRowChunks;
  const uint16_t* k = p.k + token * p.k_token;
  const uint16_t* v = p.v + token * p.v_token;
  uint4 kx[4], vx[4];
  auto load = [&](int first) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int c = first + 32 * i + lane;
      if (c < chunks) {
        kx[i] = __ldcs(reinterpret_cast<const uint4*>(k + (c / kRowChunks) * p.k_head + (c % kRowChunks) * 8));
        vx[i] = __ldcs(reinterpret_cast<const uint4*>(v + (c / kRowChunks) * p.v_head + (c % kRowChunks) * 8));
      }
    }
  };
  load(0);
  const int seq = last_not_above(p.cache.batch, token, [&](int b) { return __ldcg(p.cu + b); });
  const int2 rows = sequence_rows(p.cu, seq, p.total, p.status, 6);
  if (token < rows.x || token >= rows.y) return;   // behind the last sequence
  const int place = max(__ldcg(p.cache.lens + seq), 0) - (rows.y - token);
  const int page = page_of(p.cache, seq, place >> p.cache.page_shift, p.status, 7);
  if (page < 0) return;
  const int at = place & ((1 << p.cache.page_shift) - 1);
  uint16_t* k_to = p.cache.k + page * p.cache.k_page + at * p.cache.k_place;
  uint16_t* v_to = p.cache.v + page * p.cache.v_page + at * p.cache.v_place;
  for (int first = 0;;) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int c = first + 32 * i + lane;
      if (c < chunks) {
        *reinterpret_cast<uint4*>(k_to + (c / kRowChunks) * p.cache.k_head + (c % kRowChunks) * 8) = kx[i];
        *reinterpret_cast<uint4*>(v_to + (c / kRowChunks) * p.cache.v_head + (c % kRowChunks) * 8) = vx[i];
      }
    }
    first += 128;
    if (first >= chunks) break;
    load(first);
  }
}

// ------------------------------------------------------------------------------------------
// Eviction, first half: which keys stay. A cluster of CTAs ranks one row (sequence, key-value head), each CTA a run of its
// candidates (all but the `recent` last keys): radix selection of the (keep - recent)-th largest mass, 11 + 11 + 10 bits, over
// histograms that the CTAs of the cluster read from each other; then every warp counts and writes out its share in order.
// ------------------------------------------------------------------------------------------
constexpr int kSelectThreads = 1024;
constexpr int kSelectWarps = kSelectThreads / 32;
constexpr int kBins = 2048;
constexpr int kCachedKeys = 24 * 1024;   // of a CTA's run, held in shared memory (96 KB) as ordered keys

struct EvictSmem {
  int hist[kBins];
  int warp_sum[kSelectWarps];
  int found_bin, found_above;
  int above[kSelectWarps], equal[kSelectWarps];   // keys above / equal to the threshold in each warp's share
  int cta_above, cta_equal;
  uint32_t keys[kCachedKeys];
};

__global__ void __launch_bounds__(kSelectThreads) evict_select_kernel(const EvictParams p) {
  namespace cg = cooperative_groups;
  extern __shared__ __align__(16) uint8_t smem_raw[];
  EvictSmem& sm = *reinterpret_cast<EvictSmem*>(smem_raw);
  wait_for_previous_kernel();
  cg::cluster_group cluster = cg::this_cluster();
  const int ranks = static_cast<int>(cluster.num_blocks()), rank = static_cast<int>(cluster.block_rank());
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
  for (int j = me; j < p.recent; j += all) {
    kept[need + j] = candidates + j;
    mass_out[need + j] = __ldcg(mass + candidates + j);
  }
  if (need == 0) return;
  // this CTA's run of candidates, in whole warps' shares
  const int share = (candidates + ranks * kSelectWarps - 1) / (ranks * kSelectWarps);   // candidates per warp
  const int run0 = min(rank * kSelectWarps * share, candidates), run1 = min((rank + 1) * kSelectWarps * share, candidates);
  const int run = run1 - run0;
  for (int i = tid; i < min(run, kCachedKeys); i += kSelectThreads) sm.keys[i] = ordered_key(__ldcg(mass + run0 + i));
  auto key_at = [&](int i) -> uint32_t { return i < kCachedKeys ? sm.keys[i] : ordered_key(__ldcg(mass + run0 + i)); };
  // ---- the threshold -----------------------------------------------------------------------
  uint32_t prefix = 0u;
  int left = need;          // of the keys that agree with `prefix` in the bits decided so far
  for (int step = 0; step < 3; ++step) {
    const int shift = step == 0 ? 21 : (step == 1 ? 10 : 0);
    const int bins = step == 2 ? 1024 : kBins;
    for (int i = tid; i < kBins; i += kSelectThreads) sm.hist[i] = 0;
    __syncthreads();
    for (int i = tid; i < run; i += kSelectThreads) {
      const uint32_t key = key_at(i);
      const bool in = step == 0 || (step == 1 ? (key >> 21) == (prefix >> 21) : (key >> 10) == (prefix >> 10));
      if (in) atomicAdd(&sm.hist[(key >> shift) & (bins - 1)], 1);
    }
    cluster.sync();
    // bins from the top down, two to a thread: sums over the cluster, then a scan over the CTA
    const int hi_bin = kBins - 1 - 2 * tid, lo_bin = hi_bin - 1;
    int in_hi = 0, in_lo = 0;
    for (int r = 0; r < ranks; ++r) {
      const int2 two = *reinterpret_cast<const int2*>(cluster.map_shared_rank(&sm.hist[lo_bin], r));
      in_lo += two.x;
      in_hi += two.y;
    }
    int sum = in_hi + in_lo;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
      const int other = __shfl_up_sync(0xffffffffu, sum, d);
      if (lane >= d) sum += other;
    }
    if (lane == 31) sm.warp_sum[warp] = sum;
    __syncthreads();
    int before = 0;
    for (int w = 0; w < warp; ++w) before += sm.warp_sum[w];
    const int above_lo = before + sum - in_lo, above_hi = above_lo - in_hi;   // keys in the bins above each of the two
    if (above_hi < left && above_hi + in_hi >= left) {
      sm.found_bin = hi_bin;
      sm.found_above = above_hi;
    }
    if (above_lo < left && above_lo + in_lo >= left) {
      sm.found_bin = lo_bin;
      sm.found_above = above_lo;
    }
    cluster.sync();   // (the histograms have been read; found_* are visible)
    prefix |= static_cast<uint32_t>(sm.found_bin) << shift;
    left -= sm.found_above;
    __syncthreads();
  }
  // Kept: keys above `prefix`, and the first `left` of those equal to it.
  // ---- where each warp's share goes ----------------------------------------------------------
  const int my0 = min(warp * share, run), my1 = min(my0 + share, run);
  int above = 0, equal = 0;
  for (int i = my0 + lane; i < my1; i += 32) {
    const uint32_t key = key_at(i);
    above += key > prefix;
    equal += key == prefix;
  }
  above = __reduce_add_sync(0xffffffffu, above);
  equal = __reduce_add_sync(0xffffffffu, equal);
  if (lane == 0) {
    sm.above[warp] = above;
    sm.equal[warp] = equal;
  }
  __syncthreads();
  if (warp == 0) {
    const int a = __reduce_add_sync(0xffffffffu, sm.above[lane]), e = __reduce_add_sync(0xffffffffu, sm.equal[lane]);
    if (lane == 0) {
      sm.cta_above = a;
      sm.cta_equal = e;
    }
  }
  cluster.sync();
  int above_before = 0, equal_before = 0;   // in the shares before this warp's
  for (int r = 0; r < rank; ++r) {
    above_before += *cluster.map_shared_rank(&sm.cta_above, r);
    equal_before += *cluster.map_shared_rank(&sm.cta_equal, r);
  }
  for (int w = 0; w < warp; ++w) {
    above_before += sm.above[w];
    equal_before += sm.equal[w];
  }
  for (int i0 = my0; i0 < my1; i0 += 32) {
    const int i = i0 + lane;
    const uint32_t key = i < my1 ? key_at(i) : 0u;
    const bool is_above = i < my1 && key > prefix, is_equal = i < my1 && key == prefix;
    const uint32_t lower = (1u << lane) - 1u;
    const uint32_t a = __ballot_sync(0xffffffffu, is_above), e = __ballot_sync(0xffffffffu, is_equal);
    const int my_equal = equal_before + __popc(e & lower);
    if (is_above || (is_equal && my_equal < left)) {
      const int at = above_before + __popc(a & lower) + min(my_equal, left);
      kept[at] = run0 + i;
      mass_out[at] = __ldcg(mass + run0 + i);
    }
    above_before += __popc(a);
    equal_before += __popc(e);
  }
  cluster.sync();   // no CTA leaves while another may still read its counts
}

// ------------------------------------------------------------------------------------------
// Eviction, second half: the kept rows of K and V to their new pages. Sixteen threads move a row; each has four rows of K and V
// in flight.
// ------------------------------------------------------------------------------------------
constexpr int kMoveThreads = 256;
constexpr int kMoveRows = 4;    // per sixteen threads
constexpr int kMoveCta = kMoveThreads / 16 * kMoveRows;

__global__ void __launch_bounds__(kMoveThreads) evict_move_kernel(const EvictParams p) {
  wait_for_previous_kernel();
  const int ctas_per_row = (p.keep + kMoveCta - 1) / kMoveCta;
  const int row = blockIdx.x / ctas_per_row, first = (blockIdx.x - row * ctas_per_row) * kMoveCta;
  const int seq = row / p.from.heads_kv, head = row % p.from.heads_kv;
  const int part = threadIdx.x >> 4, c = (threadIdx.x & 15) * 8;
  const int32_t* kept = p.kept + static_cast<int64_t>(row) * p.keep;
  uint4 kx[kMoveRows], vx[kMoveRows];
  int from[kMoveRows];
#pragma unroll
  for (int i = 0; i < kMoveRows; ++i) {
    const int j = first + i * (kMoveThreads / 16) + part;
    from[i] = j < p.keep ? __ldcg(kept + j) : -1;
  }
#pragma unroll
  for (int i = 0; i < kMoveRows; ++i) {
    kx[i] = vx[i] = make_uint4(0u, 0u, 0u, 0u);
    if (from[i] >= 0) {
      const int page = page_of(p.from, seq, from[i] >> p.from.page_shift, p.status, 9);
      const int at = from[i] & ((1 << p.from.page_shift) - 1);
      if (page >= 0) {
        kx[i] = __ldcs(reinterpret_cast<const uint4*>(p.from.k + page * p.from.k_page + at * p.from.k_place + head * p.from.k_head + c));
        vx[i] = __ldcs(reinterpret_cast<const uint4*>(p.from.v + page * p.from.v_page + at * p.from.v_place + head * p.from.v_head + c));
      }
    }
  }
#pragma unroll
  for (int i = 0; i < kMoveRows; ++i) {
    const int j = first + i * (kMoveThreads / 16) + part;
    if (from[i] >= 0) {
      const int page = page_of(p.to, seq, j >> p.to.page_shift, p.status, 10);
      const int at = j & ((1 << p.to.page_shift) - 1);
      if (page >= 0) {
        *reinterpret_cast<uint4*>(p.to.k + page * p.to.k_page + at * p.to.k_place + head * p.to.k_head + c) = kx[i];
        *reinterpret_cast<uint4*>(p.to.v + page * p.to.v_page + at * p.to.v_place + head * p.to.v_head + c) = vx[i];
      }
    }
  }
}

}  // namespace

cudaError_t launch_cache_write(const CacheWriteParams& p, cudaStream_t stream) {
  const int ctas = (p.total + kWriteWarps - 1) / kWriteWarps;
  return launch_overlapped(cache_write_kernel, ctas, ctas, 32 * kWriteWarps, 0, stream, p);
}

cudaError_t launch_cache_evict(const EvictParams& p, cudaStream_t stream) {
  const int rows = p.from.batch * p.from.heads_kv;
  const int smem = static_cast<int>(sizeof(EvictSmem));
  static SmemLimit limit;
  cudaError_t e = ensure_dynamic_smem(evict_select_kernel, smem, limit);
  if (e != cudaSuccess) return e;
  // As many CTAs to a row as fill the device, up to the portable cluster size, for rows long enough to be shared.
  const int room = p.from.max_pages << p.from.page_shift;
  int ranks = 1;
  while (ranks < 8 && rows * ranks * 2 <= 148 && room / (2 * ranks) >= 2048) ranks *= 2;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(rows * ranks));
  cfg.blockDim = dim3(kSelectThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2] = {};
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = static_cast<unsigned>(ranks);
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  e = cudaLaunchKernelEx(&cfg, evict_select_kernel, p);
  if (e == cudaSuccess) {
    cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>((p.keep + kMoveCta - 1) / kMoveCta * rows));
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
