// Attention of one new token per sequence over a paged key-value cache, head_dim 128, bf16 or fp16, fp32 softmax.
//
// Every cached key and value is read once (with more than 16 query heads in a group once for every 16 of them) and used for
// these few heads only, so HBM bounds it: what matters is that every SM keeps loads in flight all the time, whatever the
// lengths are. A warp takes 16 keys at a time: one TMA instruction brings their K (4 KB), one their V, each into a place
// that only this warp reads, and the next one is issued as soon as the warp has the current one in registers. 16 warps an
// SM, 128 KB on their way. (Measured on this pattern alone, 2.8 GB: TMA 6.9 TB/s with 64 to 192 KB on their way, 16-byte
// loads into registers 6.8, cp.async 5.2. As loads into registers the whole kernel took 436 us for 24 x 7000 keys x 32
// heads, its accumulators leaving no room for the tiles.)
//   S^T [16 keys x 8 heads]  = K [16 x 128] Q^T: mma.m16n8k16 with K as the A operand. A dot product does not care in which
//     order it takes head_dim, so a thread's A fragments of two k-steps are one 16-byte piece of a key row, and Q is read with
//     the same permutation.
//   O^T [128 x 8 heads] += V^T P^T: V^T as the A operand needs pairs of keys at one d; a thread reads 16-byte pieces of four
//     keys and pairs them up with byte permutes, d running over the rows of the eight m-tiles in the order that falls out.
//   P^T is S^T's accumulator turned around in registers (movmatrix).
// (The fifth-generation tensor instructions work on 128 rows, with their results in tensor memory and a barrier between each
// step: with 8 heads the legacy instructions take a tenth of the time the bytes need, and each warp goes at its own pace.)
//
// How the work is divided: a unit is 64 keys of one (sequence, key-value head), 16 for each of a CTA's four warps. All units
// of the call, in order, are dealt out to the CTAs that fit on the device in equal contiguous shares; each CTA finds its own
// in the lengths. So a long sequence is split over as many CTAs as its share of the work, many short ones share a CTA, and
// nothing depends on the longest length. A sequence's head that one CTA has from start to end is finished by it; of others,
// each CTA leaves its part (reference, sum, unnormalised O in fp32), and a second kernel, already waiting, joins the parts.
// (Smaller shares, taken over by CTAs that are done early, were slower: each costs a start and a part.)
// That kernel also adds up the keys' attention weights where asked: the first one leaves the logits (4 bytes per head and
// key against 512 per key), from which p = 2^(logit - LSE) follows once the LSE is known.
//
// Roundings: logits, sums, O and weights are fp32 throughout. P goes to the matrix instructions in the cache's 16-bit type, the
// sum of a softmax takes it unrounded: up to half a step of P, 2^-8 of a weight in bf16 and 2^-11 in fp16, with either sign, averages
// out over the keys (errors against 64 bits 2.3e-3 of O's size in bf16, most of it O's own rounding, 2.9e-4 in fp16).
//
// Measured (caches cold): 24 x 6000-8192 keys x 32 heads 416 us, 6.7 TB/s; 131072 x 8 heads 90, 5.9; 48 x 300-8000 x 4 heads
// 53, 4.4 (with weights 57); one sequence of 1500 keys x 4 heads 7.5 in a graph; 131072 x 2 heads with 32 query heads 37, with 40,
// which are two walks over 134 MB, 46. The shorter ones are bound by what comes before and after the stream of keys: lengths - page -
// first tiles, about 3 us, and the joining kernel, 4 to 8.
#include <algorithm>

#include "paged_loads.h"
#include "sequences.cuh"
#include "softmax_pipeline.cuh"

namespace sparsed {
namespace {

constexpr int kHeadDim = 128;
constexpr int kWarps = 4;
constexpr int kThreads = 32 * kWarps;
constexpr int kWarpKeys = 16;
constexpr int kUnit = kWarps * kWarpKeys;
constexpr int kTileBytes = kWarpKeys * kHeadDim * 2;
constexpr int kMostCtas = 1024;

template <class Type>
__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1);
template <>
__device__ __forceinline__ void mma16816<Bf16Type>(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                                   uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
template <>
__device__ __forceinline__ void mma16816<Fp16Type>(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                                   uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// An 8 x 8 matrix of 16-bit numbers (thread 4 r + c holds row r, columns 2 c and 2 c + 1), turned around.
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

__device__ __forceinline__ void load_shared(uint32_t* x, uint32_t from) {
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]) : "r"(from) : "memory");
}

__device__ __forceinline__ int units_of(int len) { return (len + kUnit - 1) / kUnit; }

// CTAs of the main kernel on an SM, by its registers (128 / 168) and shared memory (54 / 60 KB).
__host__ __device__ constexpr int ctas_per_sm(int heads) { return heads == 8 ? 4 : 3; }

// kHeads: query heads a CTA works on at once, 8 or 16 (the n-tiles of the matrix instructions).
template <int kHeads>
struct PagedSmem {
  // K and V of each warp's 16 keys: two 64-wide halves of head_dim, rows of 128 bytes, 128-byte swizzle
  alignas(1024) uint8_t tiles[kWarps][2][kTileBytes];
  alignas(16) uint16_t q[2][kHeads][160];   // rows 320 bytes apart: two rows' pieces fall on different banks
  alignas(16) float o[kWarps][8][kHeadDim + 4];   // of one n-tile
  float m[kWarps][kHeads], l[kWarps][kHeads];
  uint64_t full[kWarps][2];
  int warp_units[kWarps];
  int found_seq, found_units, found_len;
  int abort_flag;
};

template <class Type, int kHeads, bool kMass>
__global__ void __launch_bounds__(kThreads, ctas_per_sm(kHeads))
attn_paged_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v, const PagedParams p) {
  constexpr int kNT = kHeads / 8;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  PagedSmem<kHeads>& sm = *reinterpret_cast<PagedSmem<kHeads>*>(smem_raw);
  wait_for_previous_kernel(!p.fills);
  if ((smem_u32(smem_raw) & 1023u) != 0u) {
    if (threadIdx.x == 0) record_status(p.status, 2, 5);
    return;
  }
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
  // Row g of the 16 x 128 operand K holds key `spread` of its eight, and row g of V^T holds head_dim 8 * spread + j: with this
  // order neither reading of the swizzled tiles meets a bank conflict.
  const int spread = (g >> 1) | ((g & 1) << 2);
  const CacheView& c = p.cache;
  const int head_chunks = (p.group + kHeads - 1) / kHeads;
  const int rows = c.heads_kv * head_chunks;   // (key-value head, chunk of its query heads) pairs per sequence

  // ---- this CTA's share: a scan over the lengths ------------------------------------------------
  const int per_thread = (c.batch + kThreads - 1) / kThreads;
  const int b0 = min(tid * per_thread, c.batch), b1 = min(b0 + per_thread, c.batch);
  int mine = 0, last_len = 0;
  for (int b = b0; b < b1; ++b) {
    last_len = cached_length(c, b, p.status, 11);
    mine += units_of(last_len);
  }
  int sum = mine;
#pragma unroll
  for (int d = 1; d < 32; d *= 2) {
    const int other = __shfl_up_sync(0xffffffffu, sum, d);
    if (lane >= d) sum += other;
  }
  if (lane == 31) sm.warp_units[warp] = sum;
  if (tid == 0) {
    sm.found_seq = sm.found_units = sm.found_len = 0;   // (always found, unless the lengths change under the call)
    sm.abort_flag = 0;
  }
  if (lane < 2) mbar_init(&sm.full[warp][lane], 1);
  mbar_fence_init();
  __syncthreads();
  int before = sum - mine, total = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    if (w < warp) before += sm.warp_units[w];
    total += sm.warp_units[w];
  }
  if (blockIdx.x == 0) {   // for the joining kernel
    int at = before;
    for (int b = b0; b < b1; ++b) {
      p.prefix[b] = at;
      at += units_of(cached_length(c, b, p.status, 11));
    }
    if (tid == 0) p.prefix[c.batch] = total;
  }
  const int all_units = total * rows;
  const int share = (all_units + p.ctas - 1) / p.ctas;
  const int unit0 = static_cast<int>(blockIdx.x) * share, unit1 = min(unit0 + share, all_units);
  if (unit0 >= unit1) return;
  {
    const int u = unit0 / rows;   // `rows` times a sequence's units lie together, so unit0 is in the sequence that has u
    if (before <= u && u < before + mine) {
      int at = before, b = b0;
      if (per_thread > 1) {   // (one sequence to a thread: it is at hand)
        for (; b < b1; ++b) {
          last_len = cached_length(c, b, p.status, 11);
          if (u < at + units_of(last_len)) break;
          at += units_of(last_len);
        }
      }
      sm.found_seq = b;
      sm.found_units = at;
      sm.found_len = last_len;
    }
  }
  __syncthreads();

  // ---- the segments of the share: units of one sequence and row each --------------------------------
  int unit = unit0, seq = sm.found_seq, len = sm.found_len, n_units = units_of(len);
  int seq_unit0 = sm.found_units * rows;   // the sequence's first unit
  int tile0 = 0, tile1 = 0, kv_head = 0, head0 = 0, heads = 0;
  int page = -1, next_page = -1;   // of this warp's keys of units `tile` and `tile` + 1; -1: nothing to do there
  uint32_t uses = 0;               // tiles this warp has worked on: the phase of its barriers
  uint32_t buf = 0;                // of Q
  const int place_mask = (1 << c.page_shift) - 1;
  const uint64_t once = l2_evict_first();   // (so that the logits and parts for the joining kernel stay in L2)
  const uint32_t k_tile = smem_u32(sm.tiles[warp][0]), v_tile = smem_u32(sm.tiles[warp][1]);

  // Positions [key0, key0 + 16) are this warp's of a unit. They lie in one page (page sizes are multiples of 16).
  auto page_at = [&](int tile) -> int {
    const int key0 = tile * kUnit + warp * kWarpKeys;
    return tile < tile1 && key0 < len ? page_of(c, seq, key0 >> c.page_shift, p.status, 12) : -1;
  };
  // K (0) or V (1) of this warp's keys in a unit on its way, by one lane, after all lanes have read what was there. The reads are
  // ordinary ones and the copy is not: without the fence, keys that are in L2 can land before the last of the reads is done.
  auto load = [&](int which, int tile, int at_page) {
    fence_proxy_async_smem();
    __syncwarp();
    if (at_page >= 0 && lane == 0) {
      mbar_expect_tx(&sm.full[warp][which], kTileBytes);
      tma_load_5d(sm.tiles[warp][which], which == 0 ? &tm_k : &tm_v, &sm.full[warp][which], 0,
                  (tile * kUnit + warp * kWarpKeys) & place_mask, 0, kv_head, at_page, once);
    }
  };
  // finds the segment that begins at `unit` and sends its first loads off
  auto begin_segment = [&]() {
    while (unit >= seq_unit0 + n_units * rows && seq + 1 < c.batch) {   // on to the next sequence that has any
      seq_unit0 += n_units * rows;
      ++seq;
      len = cached_length(c, seq, p.status, 11);
      n_units = units_of(len);
    }
    const int row = n_units > 0 ? (unit - seq_unit0) / n_units : 0;
    tile0 = unit - seq_unit0 - row * n_units;
    tile1 = min(n_units, tile0 + unit1 - unit);
    kv_head = row / head_chunks;
    head0 = kv_head * p.group + (row - kv_head * head_chunks) * kHeads;
    heads = min(kHeads, (kv_head + 1) * p.group - head0);   // of this chunk
    page = page_at(tile0);
    next_page = page_at(tile0 + 1);
    // Q: heads beyond the group's last are zeros
    constexpr int kPieces = kHeads * 16 / kThreads;
    uint4 qx[kPieces];
#pragma unroll
    for (int x = 0; x < kPieces; ++x) {
      const int i = x * kThreads + tid;
      qx[x] = make_uint4(0u, 0u, 0u, 0u);
      if ((i >> 4) < heads) qx[x] = __ldcg(reinterpret_cast<const uint4*>(p.q + seq * p.q_seq + (head0 + (i >> 4)) * p.q_head + (i & 15) * 8));
    }
    load(0, tile0, page);
    load(1, tile0, page);
#pragma unroll
    for (int x = 0; x < kPieces; ++x) {
      const int i = x * kThreads + tid;
      *reinterpret_cast<uint4*>(&sm.q[buf][i >> 4][(i & 15) * 8]) = qx[x];
    }
  };

  begin_segment();
  bool ok = true;
  // A wait has run out: what this warp has on its way must have landed before the CTA leaves (bounded like every wait).
  auto drain = [&](PagedWait failed) {
    const PagedLoads loads = paged_loads_on_their_way(failed, uses, next_page >= 0);
    for (uint32_t i = 0; loads.keys && i < kSpinLimit && !mbar_try_wait(&sm.full[warp][0], loads.keys_use & 1); ++i) {
    }
    for (uint32_t i = 0; loads.values && i < kSpinLimit && !mbar_try_wait(&sm.full[warp][1], loads.values_use & 1); ++i) {
    }
  };
  while (true) {
    float o[kNT][8][4];
    float m[kNT][2], l[kNT][2];
#pragma unroll
    for (int n = 0; n < kNT; ++n) {
#pragma unroll
      for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int x = 0; x < 4; ++x) o[n][j][x] = 0.f;
      m[n][0] = m[n][1] = -INFINITY;
      l[n][0] = l[n][1] = 0.f;
    }
    const int64_t room = static_cast<int64_t>(c.max_pages) << c.page_shift;   // logits per query head
    [[maybe_unused]] float* logits = nullptr;   // of key `spread`, head 2t
    if constexpr (kMass) logits = p.logits + (static_cast<int64_t>(seq) * c.heads_kv * p.group + head0 + 2 * t) * room + spread;
    __syncthreads();   // Q is there
    for (int tile = tile0; tile < tile1; ++tile) {
      const int key0 = tile * kUnit + warp * kWarpKeys;
      const int page_after = page_at(tile + 2);
      if (page >= 0) {   // (the same for the whole warp; false: no keys, or no page)
        // ---- S^T = K Q^T, in two chains of dependent instructions
        float s[kNT][4];
        {
          ok = mbar_wait(&sm.full[warp][0], uses & 1, &sm.abort_flag, p.status, 15);
          if (!(ok = __all_sync(0xffffffffu, ok))) {
            drain(PagedWait::kKeys);
            break;
          }
          uint32_t kx[2][16];   // rows g and g + 8, pieces 4 i + t
          const uint32_t at = k_tile + spread * 128 + ((t ^ spread) << 4);
#pragma unroll
          for (int r = 0; r < 2; ++r)
#pragma unroll
            for (int i = 0; i < 4; ++i) load_shared(kx[r] + 4 * i, (at ^ ((i & 1) << 6)) + r * 1024 + (i >> 1) * 2048);
          load(0, tile + 1, next_page);
#pragma unroll
          for (int n = 0; n < kNT; ++n) {
            float s2[4] = {0.f, 0.f, 0.f, 0.f};
            s[n][0] = s[n][1] = s[n][2] = s[n][3] = 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const uint4 q = *reinterpret_cast<const uint4*>(&sm.q[buf][n * 8 + g][(4 * i + t) * 8]);
              mma16816<Type>(s[n], kx[0][4 * i], kx[1][4 * i], kx[0][4 * i + 1], kx[1][4 * i + 1], q.x, q.y);
              mma16816<Type>(s2, kx[0][4 * i + 2], kx[1][4 * i + 2], kx[0][4 * i + 3], kx[1][4 * i + 3], q.z, q.w);
            }
#pragma unroll
            for (int x = 0; x < 4; ++x) s[n][x] = (s[n][x] + s2[x]) * p.scale_log2;
          }
        }
        // ---- probabilities
        const int valid = len - key0;
        if (valid < kWarpKeys) {
#pragma unroll
          for (int n = 0; n < kNT; ++n)
#pragma unroll
            for (int x = 0; x < 4; ++x)
              if (spread + 8 * (x >> 1) >= valid) s[n][x] = -INFINITY;
        }
        bool outgrown = false;
#pragma unroll
        for (int n = 0; n < kNT; ++n)
#pragma unroll
          for (int x = 0; x < 2; ++x) outgrown = outgrown || fmaxf(s[n][x], s[n][x + 2]) > m[n][x] + Type::kSlack;
        if constexpr (kMass) {
#pragma unroll
          for (int n = 0; n < kNT; ++n)
#pragma unroll
            for (int x = 0; x < 4; ++x)
              if (8 * n + 2 * t + (x & 1) < heads && spread + 8 * (x >> 1) < valid)
                logits[(8 * n + (x & 1)) * room + key0 + 8 * (x >> 1)] = s[n][x];
        }
        if (__any_sync(0xffffffffu, outgrown)) {
          // logits well above their head's reference (or there is none yet): the tile's maximum, less the headroom, becomes the reference
#pragma unroll
          for (int n = 0; n < kNT; ++n)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              float top = fmaxf(s[n][x], s[n][x + 2]);
              top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 4));
              top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 8));
              top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 16));
              if (top > m[n][x] + Type::kSlack) {   // (a head's result does not depend on the other heads)
                top -= Type::kHeadroom;
                const float alpha = fast_exp2(m[n][x] - top);   // 0 when nothing was accumulated yet
                m[n][x] = top;
                l[n][x] *= alpha;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                  o[n][j][x] *= alpha;
                  o[n][j][x + 2] *= alpha;
                }
              }
            }
        }
        uint32_t pt[kNT][2];   // P^T as the B operand: rows 2t, 2t + 1 / 2t + 8, 2t + 9 of S^T, head g
#pragma unroll
        for (int n = 0; n < kNT; ++n) {
          float e[4];
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            const float ref = m[n][x & 1] == -INFINITY ? 0.f : m[n][x & 1];   // (only logits of -inf so far)
            e[x] = fast_exp2(s[n][x] - ref);
            l[n][x & 1] += e[x];
          }
          pt[n][0] = transpose8x8(Type::pack(e[0], e[1]));
          pt[n][1] = transpose8x8(Type::pack(e[2], e[3]));
        }
        // ---- O^T += V^T P^T. Rows 2t, 2t + 1, 2t + 8, 2t + 9 of S^T are keys t, t + 4, t + 8, t + 12.
        ok = mbar_wait(&sm.full[warp][1], uses & 1, &sm.abort_flag, p.status, 16);
        if (!(ok = __all_sync(0xffffffffu, ok))) {
          drain(PagedWait::kValues);
          break;
        }
        uint32_t vx[4][8];   // pieces `spread` and `spread` + 8 of the four keys
        const uint32_t at = v_tile + t * 128 + ((spread ^ t) << 4);
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int i = 0; i < 2; ++i) load_shared(vx[r] + 4 * i, (at ^ ((r & 1) << 6)) + r * 512 + i * 2048);
        load(1, tile + 1, next_page);
        if (valid < kWarpKeys) {   // what lies behind the sequence may be anything, and 0 * NaN is NaN
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (t + 4 * r >= valid) {
#pragma unroll
              for (int i = 0; i < 8; ++i) vx[r][i] = 0u;
            }
        }
#pragma unroll
        for (int w = 0; w < 4; ++w)
#pragma unroll
          for (int odd = 0; odd < 2; ++odd) {
            const uint32_t sel = odd ? 0x7632u : 0x5410u;
            const uint32_t a0 = __byte_perm(vx[0][w], vx[1][w], sel), a1 = __byte_perm(vx[0][4 + w], vx[1][4 + w], sel);
            const uint32_t a2 = __byte_perm(vx[2][w], vx[3][w], sel), a3 = __byte_perm(vx[2][4 + w], vx[3][4 + w], sel);
#pragma unroll
            for (int n = 0; n < kNT; ++n) mma16816<Type>(o[n][2 * w + odd], a0, a1, a2, a3, pt[n][0], pt[n][1]);
          }
        ++uses;
      } else {
        load(0, tile + 1, next_page);
        load(1, tile + 1, next_page);
        if constexpr (kMass) {   // keys without a page have no weight
#pragma unroll
          for (int n = 0; n < kNT; ++n)
#pragma unroll
            for (int x = 0; x < 4; ++x)
              if (8 * n + 2 * t + (x & 1) < heads && key0 + spread + 8 * (x >> 1) < len)
                logits[(8 * n + (x & 1)) * room + key0 + 8 * (x >> 1)] = -INFINITY;
        }
      }
      page = next_page;
      next_page = page_after;
    }
    if (!__syncthreads_and(ok)) break;   // (a wait has run out)

    // ---- the next segment's first loads on their way, then the four warps' shares of this one together ---------
    const bool whole = tile0 == 0 && tile1 == n_units;
    const int slot = 2 * static_cast<int>(blockIdx.x) + (tile0 == 0 ? 1 : 0);
    const int done_seq = seq, done_head0 = head0, done_heads = heads;
    unit += max(tile1 - tile0, 1);   // (less than one only where the lengths change under the call)
    buf ^= 1;
    if (unit < unit1) begin_segment();
    else if (p.fills) next_kernel_may_start();
    // o[n][j]: d = 8 * spread + j (0, 1) and 64 + 8 * spread + j (2, 3) of heads 2t and 2t + 1 of n-tile n
#pragma unroll
    for (int n = 0; n < kNT; ++n) {
      if (n > 0) __syncthreads();   // the n-tile before has been read
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        l[n][x] += __shfl_xor_sync(0xffffffffu, l[n][x], 4);
        l[n][x] += __shfl_xor_sync(0xffffffffu, l[n][x], 8);
        l[n][x] += __shfl_xor_sync(0xffffffffu, l[n][x], 16);
        const int h = 8 * n + 2 * t + x;
        if (g == 0) {
          sm.m[warp][h] = m[n][x];
          sm.l[warp][h] = l[n][x];
        }
        float4* low = reinterpret_cast<float4*>(&sm.o[warp][2 * t + x][8 * spread]);
        float4* high = reinterpret_cast<float4*>(&sm.o[warp][2 * t + x][64 + 8 * spread]);
        low[0] = make_float4(o[n][0][x], o[n][1][x], o[n][2][x], o[n][3][x]);
        low[1] = make_float4(o[n][4][x], o[n][5][x], o[n][6][x], o[n][7][x]);
        high[0] = make_float4(o[n][0][x + 2], o[n][1][x + 2], o[n][2][x + 2], o[n][3][x + 2]);
        high[1] = make_float4(o[n][4][x + 2], o[n][5][x + 2], o[n][6][x + 2], o[n][7][x + 2]);
      }
      __syncthreads();
      for (int h = 8 * n; h < min(8 * n + 8, done_heads); ++h) {
        float top = sm.m[0][h];
#pragma unroll
        for (int w = 1; w < kWarps; ++w) top = fmaxf(top, sm.m[w][h]);
        const float ref = top == -INFINITY ? 0.f : top;
        float sum_l = 0.f, sum_o = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
          const float f = fast_exp2(sm.m[w][h] - ref);
          sum_l += f * sm.l[w][h];
          sum_o += f * sm.o[w][h - 8 * n][tid];
        }
        if (whole) {
          const float inv = sum_l == 0.f ? 0.f : 1.f / sum_l;   // (0: every page was missing)
          p.o[done_seq * p.o_seq + (done_head0 + h) * p.o_head + tid] = static_cast<uint16_t>(Type::pack(sum_o * inv, 0.f) & 0xffffu);
          if (tid == 0) {
            const float lse2 = top + log2f(sum_l);
            p.lse2[static_cast<int64_t>(done_seq) * c.heads_kv * p.group + done_head0 + h] = lse2;
            if (p.lse != nullptr) p.lse[static_cast<int64_t>(done_seq) * c.heads_kv * p.group + done_head0 + h] = lse2 * 0.69314718055994531f;
          }
        } else {
          p.part_o[(static_cast<int64_t>(slot) * kHeads + h) * kHeadDim + tid] = sum_o;
          if (tid == 0) p.part_ml[slot * kHeads + h] = make_float2(top, sum_l);
        }
      }
    }
    // (the shares are read before any warp writes the next segment's: two barriers lie between)
    if (unit >= unit1) return;
  }
}

// ------------------------------------------------------------------------------------------
// The parts of split sequences together, and the keys' weights. Of a sequence's blocks the first ones finish some query heads
// each; with weights, the others take every so many keys of one key-value head each. How many heads and keys go by the number of
// blocks that makes (launch): each block begins with a chain of loads, so a few hundred are enough.
// ------------------------------------------------------------------------------------------
constexpr int kJoinThreads = 128;
static_assert(kJoinThreads == kHeadDim, "a thread to a number of the output");
constexpr int kJoinBatch = 8;   // parts that a warp reads at once
constexpr int kMassKeys = 4 * kJoinThreads;
constexpr int kJoinBlocks = 592;
constexpr int kMassHeads = 8;   // whose logits a thread has in flight

template <class Type, int kHeads, bool kMass>
__global__ void __launch_bounds__(kJoinThreads) join_kernel(const PagedParams p, int head_blocks, int mass_blocks) {
  __shared__ float2 warp_ml[kJoinThreads / 32];
  __shared__ float4 warp_o[kJoinThreads / 32][32];
  extern __shared__ float lse_of[];   // weights: base-2 LSE of the group's query heads
  wait_for_previous_kernel(!p.fills);
  const CacheView& c = p.cache;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int blocks_per_seq = head_blocks + c.heads_kv * mass_blocks;
  const int seq = blockIdx.x / blocks_per_seq, what = blockIdx.x - seq * blocks_per_seq;
  const int heads_q = c.heads_kv * p.group;
  const int head_chunks = (p.group + kHeads - 1) / kHeads, rows = c.heads_kv * head_chunks;
  const int first = __ldcg(p.prefix + seq), n_units = __ldcg(p.prefix + seq + 1) - first;
  const int all_units = __ldcg(p.prefix + c.batch) * rows;
  const int share = (all_units + p.ctas - 1) / p.ctas;
  // the CTAs that had query head `head`: first and last of them
  auto ctas_of = [&](int head) -> int2 {
    const int in_group = head % p.group, row = head / p.group * head_chunks + in_group / kHeads;
    const int unit0 = first * rows + row * n_units;
    return make_int2(unit0 / share, (unit0 + n_units - 1) / share);
  };
  auto slot_of = [&](int cta, int2 ctas) -> int64_t { return 2 * cta + (cta == ctas.x ? 1 : 0); };
  if (what < head_blocks) {
    for (int head = what; head < heads_q; head += head_blocks) {
      const int in_chunk = head % p.group % kHeads;
      uint16_t* o = p.o + seq * p.o_seq + head * p.o_head;
      if (n_units == 0) {
        if (tid < kHeadDim) o[tid] = 0;
        if (p.lse != nullptr && tid == 0) p.lse[static_cast<int64_t>(seq) * heads_q + head] = -INFINITY;
        continue;
      }
      const int2 ctas = ctas_of(head);
      if (ctas.x == ctas.y) continue;   // finished already
      // Warps take the parts in turn, eight at a time, a lane four numbers of the output: all loads of a batch at once.
      const int parts = ctas.y - ctas.x + 1;
      float m = -INFINITY, l = 0.f;
      float4 o4 = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int i0 = warp; i0 < parts; i0 += kJoinBatch * kJoinThreads / 32) {
        float2 ml[kJoinBatch];
        float4 x[kJoinBatch];
        float top = m;
#pragma unroll
        for (int j = 0; j < kJoinBatch; ++j) {
          const int i = i0 + j * kJoinThreads / 32;
          ml[j] = make_float2(-INFINITY, 0.f);
          x[j] = make_float4(0.f, 0.f, 0.f, 0.f);
          if (i < parts) {
            const int64_t at = slot_of(ctas.x + i, ctas) * kHeads + in_chunk;
            ml[j] = __ldcg(p.part_ml + at);
            x[j] = __ldcg(reinterpret_cast<const float4*>(p.part_o + at * kHeadDim) + lane);
          }
        }
#pragma unroll
        for (int j = 0; j < kJoinBatch; ++j) top = fmaxf(top, ml[j].x);
        const float ref = top == -INFINITY ? 0.f : top, a = fast_exp2(m - ref);
        m = top;
        l *= a;
        o4 = make_float4(o4.x * a, o4.y * a, o4.z * a, o4.w * a);
#pragma unroll
        for (int j = 0; j < kJoinBatch; ++j) {
          const float f = fast_exp2(ml[j].x - ref);
          l += f * ml[j].y;
          o4 = make_float4(o4.x + f * x[j].x, o4.y + f * x[j].y, o4.z + f * x[j].z, o4.w + f * x[j].w);
        }
      }
      if (lane == 0) warp_ml[warp] = make_float2(m, l);
      warp_o[warp][lane] = o4;
      __syncthreads();
      float top = warp_ml[0].x;
#pragma unroll
      for (int w = 1; w < kJoinThreads / 32; ++w) top = fmaxf(top, warp_ml[w].x);
      const float ref = top == -INFINITY ? 0.f : top;
      float sum_l = 0.f, sum_o = 0.f;
#pragma unroll
      for (int w = 0; w < kJoinThreads / 32; ++w) {
        const float f = fast_exp2(warp_ml[w].x - ref);
        sum_l += f * warp_ml[w].y;
        sum_o += f * reinterpret_cast<const float*>(warp_o[w])[tid];
      }
      const float inv = sum_l == 0.f ? 0.f : 1.f / sum_l;
      o[tid] = static_cast<uint16_t>(Type::pack(sum_o * inv, 0.f) & 0xffffu);
      if (p.lse != nullptr && tid == 0) p.lse[static_cast<int64_t>(seq) * heads_q + head] = (top + log2f(sum_l)) * 0.69314718055994531f;
      __syncthreads();   // the next head's shares go to the same places
    }
    return;
  }
  if constexpr (!kMass) return;
  // ---- weights: keys [first_key, first_key + kMassKeys) of one key-value head, and so on
  const int kv_head = (what - head_blocks) / mass_blocks, first_key = (what - head_blocks - kv_head * mass_blocks) * kMassKeys;
  const int len = min(cached_length(c, seq, p.status, 13), n_units * kUnit);   // (n_units * kUnit: lengths that change under the call)
  if (first_key >= len) return;
  // The first heads' logits are on their way while the heads' LSE is worked out. (A key whose page is missing has -inf there.)
  const int64_t row = static_cast<int64_t>(seq) * c.heads_kv + kv_head;
  const int64_t room = static_cast<int64_t>(c.max_pages) << c.page_shift;
  const float* logits = p.logits + row * p.group * room;
  // four consecutive keys to a thread (rows of logits are whole numbers of 64 bytes)
  const float* mass_in = p.mass_in != nullptr ? p.mass_in + row * p.mass_capacity : nullptr;
  float* mass_out = p.mass_out + row * p.mass_capacity;
  const bool aligned = p.mass_capacity % 4 == 0 && ((reinterpret_cast<uintptr_t>(p.mass_in) | reinterpret_cast<uintptr_t>(p.mass_out)) & 15) == 0;
  float4 x[kMassHeads], before;
  auto load = [&](int j, int h0) {
    if (h0 == 0) {
      before = make_float4(0.f, 0.f, 0.f, 0.f);
      if (mass_in != nullptr) {
        if (aligned && j + 4 <= len) {
          before = __ldcg(reinterpret_cast<const float4*>(mass_in + j));
        } else {
          if (j < len) before.x = __ldcg(mass_in + j);
          if (j + 1 < len) before.y = __ldcg(mass_in + j + 1);
          if (j + 2 < len) before.z = __ldcg(mass_in + j + 2);
          if (j + 3 < len) before.w = __ldcg(mass_in + j + 3);
        }
      }
    }
#pragma unroll
    for (int h = 0; h < kMassHeads; ++h) {
      x[h] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (h0 + h < p.group && j < len) x[h] = __ldcg(reinterpret_cast<const float4*>(logits + (h0 + h) * room + j));
    }
  };
  load(first_key + 4 * tid, 0);
  for (int h = warp; h < p.group; h += kJoinThreads / 32) {
    const int head = kv_head * p.group + h;
    const int2 ctas = ctas_of(head);
    float lse2;
    if (ctas.x == ctas.y) {
      lse2 = __ldcg(p.lse2 + static_cast<int64_t>(seq) * heads_q + head);
    } else {
      float m = -INFINITY, l = 0.f;
      for (int cta = ctas.x + lane; cta <= ctas.y; cta += 32) {
        const float2 ml = __ldcg(p.part_ml + slot_of(cta, ctas) * kHeads + h % kHeads);
        const float top = fmaxf(m, ml.x), ref = top == -INFINITY ? 0.f : top;
        l = l * fast_exp2(m - ref) + ml.y * fast_exp2(ml.x - ref);
        m = top;
      }
      float top = m;
#pragma unroll
      for (int d = 16; d > 0; d /= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
      const float ref = top == -INFINITY ? 0.f : top;
      l *= fast_exp2(m - ref);
#pragma unroll
      for (int d = 16; d > 0; d /= 2) l += __shfl_xor_sync(0xffffffffu, l, d);
      lse2 = top + log2f(l);
    }
    if (lane == 0) lse_of[h] = lse2 == -INFINITY ? 0.f : lse2;   // (no key at all: 2^(-inf - 0) = 0)
  }
  __syncthreads();
  for (int j = first_key + 4 * tid; j - 4 * tid < len; j += mass_blocks * kMassKeys) {
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int h0 = 0; h0 < p.group; h0 += kMassHeads) {
      if (h0 > 0) load(j, h0);
#pragma unroll
      for (int h = 0; h < kMassHeads; ++h)
        if (h0 + h < p.group) {
          const float lse2 = lse_of[h0 + h];
          sum.x += fast_exp2(x[h].x - lse2);
          sum.y += fast_exp2(x[h].y - lse2);
          sum.z += fast_exp2(x[h].z - lse2);
          sum.w += fast_exp2(x[h].w - lse2);
        }
    }
    sum = make_float4(before.x + sum.x, before.y + sum.y, before.z + sum.z, before.w + sum.w);
    load(j + mass_blocks * kMassKeys, 0);
    // (the last keys' neighbours in the row of logits may hold anything: they are not stored)
    if (aligned && j + 4 <= len) {
      *reinterpret_cast<float4*>(mass_out + j) = sum;
    } else {
      if (j < len) mass_out[j] = sum.x;
      if (j + 1 < len) mass_out[j + 1] = sum.y;
      if (j + 2 < len) mass_out[j + 2] = sum.z;
      if (j + 3 < len) mass_out[j + 3] = sum.w;
    }
  }
}

// The joining kernel is always started early. Where the main kernel fills the device (p.fills), that is when its CTAs come to their
// last segment's end, and the joining kernel in its turn does not let the next one start before it is done: the next call's main
// kernel would find SMs with joining CTAs still on them and be placed unevenly (24 x 7000 keys x 32 heads, calls back to back: 508
// us against 417). Against a joining kernel that is started when the main one is done: 48 conversations of 300 to 8000 keys x 4
// heads 56.0 -> 52.6 us, with weights 59.9 -> 56.8, 128k x 8 heads 92.7 -> 90.5.
template <class Type, int kHeads>
cudaError_t launch(const CUtensorMap& tk, const CUtensorMap& tv, const PagedParams& p, cudaStream_t stream) {
  const bool mass = p.mass_out != nullptr;
  auto kernel = mass ? attn_paged_kernel<Type, kHeads, true> : attn_paged_kernel<Type, kHeads, false>;
  const int smem = static_cast<int>(sizeof(PagedSmem<kHeads>));
  static_assert(ctas_per_sm(kHeads) * (sizeof(PagedSmem<kHeads>) + 1024) <= 228 * 1024, "CTAs per SM");
  static SmemLimit limits[2];
  cudaError_t e = ensure_dynamic_smem(kernel, smem, limits[mass ? 1 : 0]);
  if (e != cudaSuccess) return e;
  e = launch_overlapped(kernel, p.ctas, p.ctas, kThreads, smem, stream, tk, tv, p);
  if (e != cudaSuccess) return e;
  const int heads_q = p.cache.heads_kv * p.group, rows = p.cache.batch * p.cache.heads_kv;
  const int chunks = ((p.cache.max_pages << p.cache.page_shift) + kMassKeys - 1) / kMassKeys;
  // about kJoinBlocks blocks for heads, and as many for weights, where there are more heads and keys than that
  const int head_blocks = std::max(1, std::min(heads_q, kJoinBlocks / p.cache.batch));
  const int mass_blocks = mass ? std::max(1, std::min(chunks, kJoinBlocks / rows)) : 0;
  const long long blocks = static_cast<long long>(head_blocks + p.cache.heads_kv * mass_blocks) * p.cache.batch;
  return mass ? launch_overlapped(join_kernel<Type, kHeads, true>, blocks, blocks, kJoinThreads, p.group * sizeof(float), stream, p, head_blocks, mass_blocks)
              : launch_overlapped(join_kernel<Type, kHeads, false>, blocks, blocks, kJoinThreads, 0, stream, p, head_blocks, 0);
}

int heads_at_once(int group) { return group <= 8 ? 8 : 16; }
int64_t round_up(int64_t x) { return (x + 255) / 256 * 256; }

}  // namespace

int paged_max_ctas(int batch, int heads_kv, int group, int max_pages, int page_size) {
  const int heads = heads_at_once(group);
  const int64_t units = (static_cast<int64_t>(max_pages) * page_size + kUnit - 1) / kUnit * batch * heads_kv * ((group + heads - 1) / heads);
  return static_cast<int>(units < kMostCtas ? (units < 1 ? 1 : units) : kMostCtas);
}

PagedLayout paged_layout(int batch, int heads_kv, int group, int max_pages, int page_size, bool with_mass) {
  const int64_t parts = 2 * static_cast<int64_t>(paged_max_ctas(batch, heads_kv, group, max_pages, page_size)) * heads_at_once(group);
  const int64_t heads_q = static_cast<int64_t>(heads_kv) * group;
  PagedLayout at;
  at.prefix = 256;
  at.lse2 = at.prefix + round_up((batch + 1ll) * 4);
  at.part_ml = at.lse2 + round_up(batch * heads_q * 4);
  at.part_o = at.part_ml + round_up(parts * 8);
  at.logits = at.part_o + round_up(parts * kHeadDim * 4);
  at.bytes = at.logits + (with_mass ? round_up(batch * heads_q * max_pages * page_size * 4) : 0);
  return at;
}

cudaError_t launch_attn_paged(const CUtensorMap& tk, const CUtensorMap& tv, PagedParams p, int sms, bool fp16, cudaStream_t stream) {
  const int heads = heads_at_once(p.group);
  const int fit = sms * ctas_per_sm(heads);
  const int most = paged_max_ctas(p.cache.batch, p.cache.heads_kv, p.group, p.cache.max_pages, 1 << p.cache.page_shift);
  p.fills = fit <= most;
  p.ctas = p.fills ? fit : most;
  if (heads == 8) return fp16 ? launch<Fp16Type, 8>(tk, tv, p, stream) : launch<Bf16Type, 8>(tk, tv, p, stream);
  return fp16 ? launch<Fp16Type, 16>(tk, tv, p, stream) : launch<Bf16Type, 16>(tk, tv, p, stream);
}

}  // namespace sparsed
