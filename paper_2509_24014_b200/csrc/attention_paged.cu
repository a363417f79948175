// Attention of one new token per sequence over a paged key-value cache, head_dim 128, bf16 or fp16, fp32 softmax.
//
// Every cached key and value is read once and used for the few query heads of its group only, so HBM bounds it: what matters
// is that every SM keeps loads in flight all the time, whatever the lengths are. A warp takes 16 keys at a time straight from
// global memory into the registers that the matrix instructions read, with no shared memory between:
//   S^T [16 keys x 8 heads]  = K [16 x 128] Q^T: mma.m16n8k16 with K as the A operand. A dot product does not care in which
//     order it takes head_dim, so a thread's A fragments of two k-steps are one 16-byte piece of a key row, and Q is read with
//     the same permutation.
//   O^T [128 x 8 heads] += V^T P^T: V^T as the A operand needs pairs of keys at one d; a thread loads 16-byte pieces of four
//     keys and pairs them up with byte permutes, d running over the rows of the eight m-tiles in the order that falls out.
//   P^T is S^T's accumulator turned around in registers (movmatrix).
// (The fifth-generation tensor instructions read their operands from shared memory and work on 128 rows: with 8 heads, loads
// into registers need neither staging nor barriers, and the legacy instructions take a tenth of the time the bytes need.)
// While the next 16 keys' K is on its way the current ones are exponentiated, and the next V while the next S^T is computed:
// 8 KB of loads per warp, 16 warps per SM (12 with two head tiles), against about 45 KB per SM that 6.5 TB/s need.
//
// How the work is divided: a unit is 64 keys of one (sequence, key-value head), 16 for each of a CTA's four warps. All units
// of the call, in order, are dealt out to the CTAs that fit on the device in equal contiguous shares; each CTA finds its own
// in the lengths. So a long sequence is split over as many CTAs as its share of the work, many short ones share a CTA, and
// nothing depends on the longest length. A sequence's head that one CTA has from start to end is finished by it; of others,
// each CTA leaves its part (reference, sum, unnormalised O in fp32), and a second kernel, already waiting, joins the parts.
// That kernel also adds up the keys' attention weights where asked: the first one leaves the logits (4 bytes per head and
// key against 512 per key), from which p = 2^(logit - LSE) follows once the LSE is known.
#include "sequences.cuh"
#include "softmax_pipeline.cuh"

namespace sparsed {
namespace {

constexpr int kHeadDim = 128;
constexpr int kWarps = 4;
constexpr int kThreads = 32 * kWarps;
constexpr int kWarpKeys = 16;
constexpr int kUnit = kWarps * kWarpKeys;
constexpr int kMostCtas = 1024;
constexpr float kSlack = 8.f;   // a probability may outgrow its reference to 2^8 before the reference moves

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

// 16 bytes into four words. (Each byte of the cache is read by one warp only, so it need not stay in L1.)
__device__ __forceinline__ void load_once(uint32_t* x, const uint16_t* p) {
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]) : "l"(p));
}
__device__ __forceinline__ void load_once_if(uint32_t* x, const uint16_t* p, bool wanted) {
  x[0] = x[1] = x[2] = x[3] = 0u;
  if (wanted) load_once(x, p);
}

__device__ __forceinline__ int units_of(int len) { return (len + kUnit - 1) / kUnit; }

// kHeads: query heads a CTA works on at once, 8 or 16 (the n-tiles of the matrix instructions).
template <int kHeads>
struct PagedSmem {
  alignas(16) uint16_t q[kHeads][160];   // rows 320 bytes apart: two rows' pieces fall on different banks
  float m[kWarps][kHeads], l[kWarps][kHeads];
  alignas(16) float o[kWarps][kHeads][kHeadDim + 4];
  int thread_units[kThreads];
  int warp_units[kWarps];
  int found_seq, found_units;
};

template <class Type, int kHeads, bool kMass>
__global__ void __launch_bounds__(kThreads, kHeads == 8 ? 4 : 3) attn_paged_kernel(const PagedParams p) {
  constexpr int kNT = kHeads / 8;
  __shared__ PagedSmem<kHeads> sm;
  wait_for_previous_kernel();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
  const CacheView& c = p.cache;
  const int head_chunks = (p.group + kHeads - 1) / kHeads;
  const int rows = c.heads_kv * head_chunks;   // (key-value head, chunk of its query heads) pairs per sequence

  // ---- this CTA's share: a scan over the lengths ------------------------------------------------
  const int per_thread = (c.batch + kThreads - 1) / kThreads;
  const int b0 = min(tid * per_thread, c.batch), b1 = min(b0 + per_thread, c.batch);
  int mine = 0;
  for (int b = b0; b < b1; ++b) mine += units_of(cached_length(c, b, p.status, 11));
  int sum = mine;
#pragma unroll
  for (int d = 1; d < 32; d *= 2) {
    const int other = __shfl_up_sync(0xffffffffu, sum, d);
    if (lane >= d) sum += other;
  }
  if (lane == 31) sm.warp_units[warp] = sum;
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
  if (tid == 0) {   // (always found, unless the lengths change under the call)
    sm.found_seq = 0;
    sm.found_units = 0;
  }
  __syncthreads();
  {
    const int u = unit0 / rows;   // `rows` times a sequence's units lie together, so unit0 is in the sequence that has u
    if (before <= u && u < before + mine) {
      int at = before, b = b0;
      for (; b < b1; ++b) {
        const int n = units_of(cached_length(c, b, p.status, 11));
        if (u < at + n) break;
        at += n;
      }
      sm.found_seq = b;
      sm.found_units = at;
    }
  }
  __syncthreads();
  int seq = sm.found_seq;
  int seq_unit0 = sm.found_units * rows;   // the sequence's first unit

  const float scale_log2 = p.scale_log2;
  const int place_mask = (1 << c.page_shift) - 1;
  const int64_t room = static_cast<int64_t>(c.max_pages) << c.page_shift;   // logits per query head

  for (int unit = unit0; unit < unit1;) {
    // ---- a segment: units of one sequence and row -------------------------------------------
    int len = cached_length(c, seq, p.status, 11);
    int n_units = units_of(len);
    while (unit >= seq_unit0 + n_units * rows && seq + 1 < c.batch) {   // on to the next sequence that has any
      seq_unit0 += n_units * rows;
      ++seq;
      len = cached_length(c, seq, p.status, 11);
      n_units = units_of(len);
    }
    if (n_units == 0) break;   // (only if the lengths change under the call)
    const int row = (unit - seq_unit0) / n_units;
    const int tile0 = unit - seq_unit0 - row * n_units;
    const int tile1 = min(n_units, tile0 + unit1 - unit);
    const int kv_head = row / head_chunks, head0 = kv_head * p.group + (row % head_chunks) * kHeads;
    const int heads = min(kHeads, p.group - (row % head_chunks) * kHeads);   // of this chunk

    // Q: heads beyond the group's last are zeros
    for (int i = tid; i < kHeads * 16; i += kThreads) {
      uint4 x = make_uint4(0u, 0u, 0u, 0u);
      if ((i >> 4) < heads) x = __ldcg(reinterpret_cast<const uint4*>(p.q + seq * p.q_seq + (head0 + (i >> 4)) * p.q_head + (i & 15) * 8));
      *reinterpret_cast<uint4*>(&sm.q[i >> 4][(i & 15) * 8]) = x;
    }

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
    uint32_t kx[2][16], vx[4][8];   // K: rows g and g + 8, pieces 4 i + t; V: keys 2t, 2t + 1, 2t + 8, 2t + 9, pieces g and g + 8
    // Positions [key0, key0 + 16) are this warp's of a unit. They lie in one page (page sizes are multiples of 16).
    auto page_at = [&](int tile) -> int {
      const int key0 = tile * kUnit + warp * kWarpKeys;
      return tile < tile1 && key0 < len ? page_of(c, seq, key0 >> c.page_shift, p.status, 12) : -1;
    };
    const uint16_t* k_lane = c.k + kv_head * c.k_head + g * c.k_place + t * 8;
    const uint16_t* v_lane = c.v + kv_head * c.v_head + 2 * t * c.v_place + g * 8;
    // K and V of the warp's keys in a unit; positions at and beyond `valid` are not read: zeros
    auto load_k = [&](int page, int key0, int valid) {
      const uint16_t* k = k_lane + page * c.k_page + (key0 & place_mask) * c.k_place;
      if (valid >= kWarpKeys) {
#pragma unroll
        for (int r = 0; r < 2; ++r, k += 8 * c.k_place)
#pragma unroll
          for (int i = 0; i < 4; ++i) load_once(kx[r] + 4 * i, k + i * 32);
      } else {
#pragma unroll
        for (int r = 0; r < 2; ++r, k += 8 * c.k_place)
#pragma unroll
          for (int i = 0; i < 4; ++i) load_once_if(kx[r] + 4 * i, k + i * 32, g + 8 * r < valid);
      }
    };
    auto load_v = [&](int page, int key0, int valid) {
      const uint16_t* v = v_lane + page * c.v_page + (key0 & place_mask) * c.v_place;
      if (valid >= kWarpKeys) {
#pragma unroll
        for (int r = 0; r < 4; ++r, v += (r == 2 ? 7 : 1) * c.v_place) {   // keys 2t, 2t + 1, 2t + 8, 2t + 9
          load_once(vx[r], v);
          load_once(vx[r] + 4, v + 64);
        }
      } else {
#pragma unroll
        for (int r = 0; r < 4; ++r, v += (r == 2 ? 7 : 1) * c.v_place) {
          const bool wanted = 2 * t + (r & 1) + 8 * (r >> 1) < valid;
          load_once_if(vx[r], v, wanted);
          load_once_if(vx[r] + 4, v + 64, wanted);
        }
      }
    };
    // valid keys of this warp in a unit: none where there is no page
    auto valid_at = [&](int tile, int page) -> int { return page < 0 ? 0 : len - tile * kUnit - warp * kWarpKeys; };

    int page = page_at(tile0);
    int valid = valid_at(tile0, page);
    load_k(page, tile0 * kUnit + warp * kWarpKeys, valid);
    load_v(page, tile0 * kUnit + warp * kWarpKeys, valid);
    int next_page = page_at(tile0 + 1);
    [[maybe_unused]] float* logits = nullptr;   // of key 0 + g, head 2t
    if constexpr (kMass)
      logits = p.logits + (static_cast<int64_t>(seq) * c.heads_kv * p.group + head0 + 2 * t) * room + g;
    __syncthreads();   // Q is there
    for (int tile = tile0; tile < tile1; ++tile) {
      const int key0 = tile * kUnit + warp * kWarpKeys;
      const int next_valid = valid_at(tile + 1, next_page);
      // ---- S^T = K Q^T, in two chains of dependent instructions
      float s[kNT][4];
#pragma unroll
      for (int n = 0; n < kNT; ++n) {
        float s2[4] = {0.f, 0.f, 0.f, 0.f};
        s[n][0] = s[n][1] = s[n][2] = s[n][3] = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint4 q = *reinterpret_cast<const uint4*>(&sm.q[n * 8 + g][(4 * i + t) * 8]);
          mma16816<Type>(s[n], kx[0][4 * i], kx[1][4 * i], kx[0][4 * i + 1], kx[1][4 * i + 1], q.x, q.y);
          mma16816<Type>(s2, kx[0][4 * i + 2], kx[1][4 * i + 2], kx[0][4 * i + 3], kx[1][4 * i + 3], q.z, q.w);
        }
#pragma unroll
        for (int x = 0; x < 4; ++x) s[n][x] = (s[n][x] + s2[x]) * scale_log2;
      }
      if (tile + 1 < tile1) load_k(next_page, key0 + kUnit, next_valid);
      const int page_after = page_at(tile + 2);
      // ---- probabilities
      if (valid > 0) {   // (the same for the whole warp)
        if (valid < kWarpKeys) {
#pragma unroll
          for (int n = 0; n < kNT; ++n)
#pragma unroll
            for (int x = 0; x < 4; ++x)
              if (g + 8 * (x >> 1) >= valid) s[n][x] = -INFINITY;
        }
        bool outgrown = false;
#pragma unroll
        for (int n = 0; n < kNT; ++n)
#pragma unroll
          for (int x = 0; x < 2; ++x) outgrown = outgrown || fmaxf(s[n][x], s[n][x + 2]) > m[n][x] + kSlack;
        if constexpr (kMass) {
#pragma unroll
          for (int n = 0; n < kNT; ++n)
#pragma unroll
            for (int x = 0; x < 4; ++x)
              if (8 * n + 2 * t + (x & 1) < heads && g + 8 * (x >> 1) < valid)
                logits[(8 * n + (x & 1)) * room + key0 + 8 * (x >> 1)] = s[n][x];
        }
        if (__any_sync(0xffffffffu, outgrown)) {
          // logits well above their head's reference (or there is none yet): the tile's maximum becomes the reference
#pragma unroll
          for (int n = 0; n < kNT; ++n)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              float top = fmaxf(s[n][x], s[n][x + 2]);
              top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 4));
              top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 8));
              top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 16));
              if (top > m[n][x] + kSlack) {   // (a head's result does not depend on the other heads)
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
        uint32_t pt[kNT][2];   // P^T as the B operand: keys 2t, 2t + 1 / 2t + 8, 2t + 9 of head g
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
        // ---- O^T += V^T P^T
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
      }
      if (tile + 1 < tile1) load_v(next_page, key0 + kUnit, next_valid);
      valid = next_valid;
      next_page = page_after;
    }

    // ---- the four warps' shares together -----------------------------------------------------
    // o[n][j]: d = 8 g + j (0, 1) and 64 + 8 g + j (2, 3) of heads 2t and 2t + 1 of n-tile n
#pragma unroll
    for (int n = 0; n < kNT; ++n)
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
        float4* low = reinterpret_cast<float4*>(&sm.o[warp][h][8 * g]);
        float4* high = reinterpret_cast<float4*>(&sm.o[warp][h][64 + 8 * g]);
        low[0] = make_float4(o[n][0][x], o[n][1][x], o[n][2][x], o[n][3][x]);
        low[1] = make_float4(o[n][4][x], o[n][5][x], o[n][6][x], o[n][7][x]);
        high[0] = make_float4(o[n][0][x + 2], o[n][1][x + 2], o[n][2][x + 2], o[n][3][x + 2]);
        high[1] = make_float4(o[n][4][x + 2], o[n][5][x + 2], o[n][6][x + 2], o[n][7][x + 2]);
      }
    __syncthreads();
    const bool whole = tile0 == 0 && tile1 == n_units;
    const int slot = 2 * static_cast<int>(blockIdx.x) + (tile0 == 0 ? 1 : 0);
    for (int h = 0; h < heads; ++h) {
      float top = sm.m[0][h];
#pragma unroll
      for (int w = 1; w < kWarps; ++w) top = fmaxf(top, sm.m[w][h]);
      const float ref = top == -INFINITY ? 0.f : top;
      float sum_l = 0.f, sum_o = 0.f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float f = fast_exp2(sm.m[w][h] - ref);
        sum_l += f * sm.l[w][h];
        sum_o += f * sm.o[w][h][tid];
      }
      if (whole) {
        const float inv = sum_l == 0.f ? 0.f : 1.f / sum_l;   // (0: every page was missing)
        p.o[seq * p.o_seq + (head0 + h) * p.o_head + tid] = static_cast<uint16_t>(Type::pack(sum_o * inv, 0.f) & 0xffffu);
        if (tid == 0) {
          const float lse2 = top + log2f(sum_l);
          p.lse2[static_cast<int64_t>(seq) * c.heads_kv * p.group + head0 + h] = lse2;
          if (p.lse != nullptr) p.lse[static_cast<int64_t>(seq) * c.heads_kv * p.group + head0 + h] = lse2 * 0.69314718055994531f;
        }
      } else {
        p.part_o[(static_cast<int64_t>(slot) * kHeads + h) * kHeadDim + tid] = sum_o;
        if (tid == 0) p.part_ml[slot * kHeads + h] = make_float2(top, sum_l);
      }
    }
    __syncthreads();   // the next segment overwrites Q and the shares
    unit += tile1 - tile0;
  }
}

// ------------------------------------------------------------------------------------------
// The parts of split sequences together, and the keys' weights. Blocks [0, heads_q) of a sequence finish one query head each;
// with weights, the others take kMassKeys keys of one key-value head each.
// ------------------------------------------------------------------------------------------
constexpr int kJoinThreads = 128;
constexpr int kMassKeys = 1024;

template <class Type, int kHeads>
__global__ void __launch_bounds__(kJoinThreads) join_kernel(const PagedParams p, int blocks_per_seq, int mass_blocks) {
  __shared__ float2 warp_ml[kJoinThreads / 32];
  __shared__ float4 warp_o[kJoinThreads / 32][32];
  extern __shared__ float lse_of[];   // weights: base-2 LSE of the group's query heads
  wait_for_previous_kernel();
  const CacheView& c = p.cache;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int seq = blockIdx.x / blocks_per_seq, what = blockIdx.x % blocks_per_seq;
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
  if (what < heads_q) {
    const int head = what, in_chunk = head % p.group % kHeads;
    uint16_t* o = p.o + seq * p.o_seq + head * p.o_head;
    if (n_units == 0) {
      o[tid] = 0;
      if (p.lse != nullptr && tid == 0) p.lse[static_cast<int64_t>(seq) * heads_q + head] = -INFINITY;
      return;
    }
    const int2 ctas = ctas_of(head);
    if (ctas.x == ctas.y) return;   // finished already
    // each warp takes every fourth part; a lane has four numbers of the output
    float m = -INFINITY, l = 0.f;
    float4 o4 = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int cta = ctas.x + warp; cta <= ctas.y; cta += kJoinThreads / 32) {
      const int64_t at = slot_of(cta, ctas) * kHeads + in_chunk;
      const float2 ml = __ldcg(p.part_ml + at);
      const float4 x = __ldcg(reinterpret_cast<const float4*>(p.part_o + at * kHeadDim) + lane);
      const float top = fmaxf(m, ml.x), ref = top == -INFINITY ? 0.f : top;
      const float a = fast_exp2(m - ref), b = fast_exp2(ml.x - ref);
      m = top;
      l = l * a + ml.y * b;
      o4 = make_float4(o4.x * a + x.x * b, o4.y * a + x.y * b, o4.z * a + x.z * b, o4.w * a + x.w * b);
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
    return;
  }
  // ---- weights of keys [key0, key0 + kMassKeys) of one key-value head
  const int kv_head = (what - heads_q) / mass_blocks, key0 = (what - heads_q) % mass_blocks * kMassKeys;
  const int len = cached_length(c, seq, p.status, 13);
  if (key0 >= len) return;
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
    if (lane == 0) lse_of[h] = lse2;
  }
  __syncthreads();
  const int64_t row = static_cast<int64_t>(seq) * c.heads_kv + kv_head;
  const int64_t room = static_cast<int64_t>(c.max_pages) << c.page_shift;
  const float* logits = p.logits + row * p.group * room;
  for (int j = key0 + tid; j < min(key0 + kMassKeys, len); j += kJoinThreads) {
    float sum = 0.f;
    const int page = page_of(c, seq, j >> c.page_shift, p.status, 12);   // (a key whose page is missing has no weight)
    if (page >= 0)
      for (int h = 0; h < p.group; ++h) sum += fast_exp2(__ldcg(logits + h * room + j) - lse_of[h]);
    const float had = p.mass_in != nullptr ? __ldcg(p.mass_in + row * p.mass_capacity + j) : 0.f;
    p.mass_out[row * p.mass_capacity + j] = had + sum;
  }
}

template <class Type, int kHeads>
cudaError_t launch(const PagedParams& p, cudaStream_t stream) {
  cudaError_t e = p.mass_out != nullptr
                      ? launch_overlapped(attn_paged_kernel<Type, kHeads, true>, p.ctas, p.ctas, kThreads, 0, stream, p)
                      : launch_overlapped(attn_paged_kernel<Type, kHeads, false>, p.ctas, p.ctas, kThreads, 0, stream, p);
  if (e != cudaSuccess) return e;
  const int room = p.cache.max_pages << p.cache.page_shift;
  const int mass_blocks = p.mass_out != nullptr ? (room + kMassKeys - 1) / kMassKeys : 0;
  const int blocks_per_seq = p.cache.heads_kv * (p.group + mass_blocks);
  const long long blocks = static_cast<long long>(blocks_per_seq) * p.cache.batch;
  return launch_overlapped(join_kernel<Type, kHeads>, blocks, blocks, kJoinThreads, p.group * sizeof(float), stream, p, blocks_per_seq, mass_blocks);
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

cudaError_t launch_attn_paged(PagedParams p, int sms, bool fp16, cudaStream_t stream) {
  const int heads = heads_at_once(p.group);
  const int fit = sms * (heads == 8 ? 4 : 3);
  const int most = paged_max_ctas(p.cache.batch, p.cache.heads_kv, p.group, p.cache.max_pages, 1 << p.cache.page_shift);
  p.ctas = fit < most ? fit : most;
  if (heads == 8) return fp16 ? launch<Fp16Type, 8>(p, stream) : launch<Bf16Type, 8>(p, stream);
  return fp16 ? launch<Fp16Type, 16>(p, stream) : launch<Bf16Type, 16>(p, stream);
}

}  // namespace sparsed
