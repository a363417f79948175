// Attention over packed sequences of different lengths, causal or not, head_dim 128, bf16 or fp16, fp32 softmax, on sm_100a.
//
// One CTA owns 128 consecutive query rows of one sequence and head and runs the pipeline of attention.cu over the sequence's
// keys, 64 at a time, up to the last one that its last row sees: a producer warp (TMA into a ring of swizzled tiles), a warp
// that issues S_t = Q K_t^T and O += P_t V_t with S, P and O in tensor memory, and four warps with a thread per query row
// (softmax_pipeline.cuh). Two CTAs per SM.
//
// Which rows: the lengths are only known on the device. Sequence b gets the tile numbers from cu_q[b] / 128 + b on: that
// leaves each sequence room for at least ceil(len / 128) tiles, ascends with b, and needs no sum over the sequences before
// it, so a CTA finds its sequence with one search in cu_q and the grid, total_q / 128 + num_seqs tiles for each head, is known
// to the host. Numbers beyond a sequence's last tile are CTAs that leave at once (at most one for each sequence and head).
//
// What a row must not see: with a causal mask the logits beyond each row's last key are set to -inf, in the tiles that the
// diagonal or the sequence's end runs through; all other tiles are walked without a comparison. P is then 0 there, but 0 * V is
// not 0 for a V that is infinite or NaN, and the tile at a sequence's end holds rows of the next sequence, or rows that nobody
// has written yet. So in those tiles the softmax threads look at V in shared memory before they hand P over: what is not
// finite becomes 0 there, and where it belongs to a key of this sequence, which some rows of the tile see, it is added to
// those rows' outputs in the epilogue, element by element.
//
// Bound: as the dense kernel, the tensor pipe and the softmax warps at the power limit; short sequences by the chain from the
// offsets to the first softmax.
#include "internal.h"
#include "sequences.cuh"
#include "softmax_pipeline.cuh"
#include "work_items.cuh"

namespace sparsed {
namespace {

constexpr int kHeadDim = 128;
constexpr int kSoftmaxThreads = 128;
constexpr int kThreads = 192;
constexpr int kTmemCols = 256;
constexpr int kColS = 0;      // two S buffers of 64 fp32 columns; P (16-bit pairs) reuses the first 32
constexpr int kColO = 128;    // O accumulator (fp32, 128 columns)
constexpr int kSlots = 5;

struct PackedSmem {
  alignas(1024) uint16_t q[2][kTileM * 64];           // two 64-wide halves of head_dim
  alignas(1024) uint16_t kv[kSlots][2][kTileN * 64];
  uint64_t q_full, kv_full[kSlots];
  uint64_t done[kSlots];   // the MMAs that read the slot have completed
  uint64_t p_full[2];
  uint32_t tmem_base;
  int abort_flag;
  int special;             // a V of this sequence in a masked tile is infinite or NaN
};

// Makes what is not finite in this thread's half row of a 64 x 128 tile of V zero. Returns whether there was any.
template <class Type>
__device__ __forceinline__ bool clean_half_row(uint16_t* half_tile, int row) {
  uint4* chunks = reinterpret_cast<uint4*>(half_tile + row * 64);
  uint32_t found = 0;
#pragma unroll
  for (int c = 0; c < 8; ++c) {
    const uint4 x = chunks[(c + row) & 7];   // (rotated: rows are 128 bytes apart; the swizzle does not matter here)
    found |= non_finite_pair<Type>(x.x) | non_finite_pair<Type>(x.y) | non_finite_pair<Type>(x.z) | non_finite_pair<Type>(x.w);
  }
  if (found == 0u) return false;
  uint32_t* words = reinterpret_cast<uint32_t*>(chunks);
  for (int i = 0; i < 32; ++i) {
    const uint32_t bad = non_finite_pair<Type>(words[i]);
    if (bad & 0x8000u) words[i] &= 0xffff0000u;
    if (bad & 0x80000000u) words[i] &= 0x0000ffffu;
  }
  return true;
}

template <class Type>
__global__ void __launch_bounds__(kThreads, 2)
attn_packed_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                   const __grid_constant__ CUtensorMap tm_v, const PackedParams p) {
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  PackedSmem& sm = *reinterpret_cast<PackedSmem*>(smem_raw);
  wait_for_previous_kernel();
  if ((smem_u32(smem_raw) & 1023u) != 0u) {
    if (threadIdx.x == 0) record_status(p.status, 2, 3);
    return;
  }
  const int tid = threadIdx.x;
  const int warp = tid >> 5;
  const int lane = tid & 31;

  // ---- which rows ------------------------------------------------------------------------
  // Heads are taken heads_per_pass at a time (their K and V stay in L2), tiles from the last one down: with a causal mask a
  // sequence's last tiles are its longest.
  const int per_pass = p.tiles * p.heads_per_pass;
  const int pass = blockIdx.x / per_pass;
  const int heads_here = min(p.heads_per_pass, p.heads_q - pass * p.heads_per_pass);
  const int in_pass = blockIdx.x - pass * per_pass;
  const int tile = p.tiles - 1 - in_pass / heads_here;
  const int head = pass * p.heads_per_pass + in_pass % heads_here;
  const int kv_head = head / p.group;
  const int seq = last_not_above(p.num_seqs, tile, [&](int b) { return __ldcg(p.cu_q + b) / kTileM + b; });
  const int2 q_rows = sequence_rows(p.cu_q, seq, p.total_q, p.status, 4);
  const int2 k_rows = sequence_rows(p.cu_k, seq, p.total_k, p.status, 5);
  const int q_len = q_rows.y - q_rows.x, k_len = k_rows.y - k_rows.x;
  const int q0 = (tile - (q_rows.x / kTileM + seq)) * kTileM;   // the CTA's first row in its sequence
  if (q0 < 0 || q0 >= q_len) return;
  const int shift = k_len - q_len;   // causal: row i sees keys up to i + shift
  const int seen = p.causal ? min(max(min(q0 + kTileM, q_len) + shift, 0), k_len) : k_len;   // keys the CTA walks
  const int num_tiles = (seen + kTileN - 1) / kTileN;
  // keys that all its rows see, in tiles: these need no mask
  const int open_tiles = (p.causal ? min(max(q0 + 1 + shift, 0), k_len) : k_len) / kTileN;

  if (num_tiles == 0) {
    // no keys: zeros, and a log-sum-exp of -inf
    for (int i = tid; i < kTileM * 16; i += kThreads) {
      const int row = q0 + (i >> 4);
      if (row < q_len)
        reinterpret_cast<uint4*>(static_cast<uint16_t*>(p.o) + (q_rows.x + row) * p.o_stride_t + head * p.o_stride_h)[i & 15] =
            make_uint4(0u, 0u, 0u, 0u);
    }
    if (p.lse != nullptr && tid < kTileM && q0 + tid < q_len)
      p.lse[static_cast<int64_t>(head) * p.total_q + q_rows.x + q0 + tid] = -INFINITY;
    return;
  }

  // ---- set-up: the producer warp starts its first loads before the CTA-wide part has finished ---------------
  auto issue_load = [&](int slot, int which, int t) {
    if (elect_one_sync()) {
      const CUtensorMap* tm = which == 0 ? &tm_k : &tm_v;
      mbar_expect_tx(&sm.kv_full[slot], kTileN * kHeadDim * 2);   // (rows beyond the tensor arrive as zeros)
      tma_load_4d(sm.kv[slot][0], tm, &sm.kv_full[slot], 0, k_rows.x + t * kTileN, kv_head, 0);
      tma_load_4d(sm.kv[slot][1], tm, &sm.kv_full[slot], 64, k_rows.x + t * kTileN, kv_head, 0);
    }
    __syncwarp();
  };
  const int early = min(2 * num_tiles, kSlots);
  if (warp == 4) {
    if (lane == 0) {
      mbar_init(&sm.q_full, 1);
      for (int s = 0; s < kSlots; ++s) mbar_init(&sm.kv_full[s], 1);
      mbar_fence_init();
    }
    __syncwarp();
    if (elect_one_sync()) {
      tma_prefetch_desc(&tm_q);
      tma_prefetch_desc(&tm_k);
      tma_prefetch_desc(&tm_v);
      mbar_expect_tx(&sm.q_full, kTileM * kHeadDim * 2);
      tma_load_4d(sm.q[0], &tm_q, &sm.q_full, 0, q_rows.x + q0, head, 0);
      tma_load_4d(sm.q[1], &tm_q, &sm.q_full, 64, q_rows.x + q0, head, 0);
    }
    __syncwarp();
    for (int i = 0; i < early; ++i) issue_load(i, i & 1, i >> 1);
  }
  if (tid == 0) {
    for (int s = 0; s < kSlots; ++s) mbar_init(&sm.done[s], 1);
    for (int s = 0; s < 2; ++s) mbar_init(&sm.p_full[s], kSoftmaxThreads);
    sm.abort_flag = 0;
    sm.special = 0;
    mbar_fence_init();
  }
  if (warp == 5) {
    tmem_alloc(&sm.tmem_base, kTmemCols);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sm.tmem_base;
  const uint32_t tO = tmem + kColO;
  int loads_issued = early;

  if (warp == 4) {
    // =============================== TMA producer =======================================
    for (int i = early; i < 2 * num_tiles; ++i) {
      const int slot = i % kSlots;
      bool ok = mbar_wait(&sm.done[slot], ((i / kSlots) - 1) & 1, &sm.abort_flag, p.status, 110);
      if (!__all_sync(0xffffffffu, ok)) break;
      issue_load(slot, i & 1, i >> 1);
      loads_issued = i + 1;
    }
  } else if (warp == 5) {
    // =============================== UMMA issuer ========================================
    const uint32_t q_lo0 = umma_desc_lo(smem_u32(sm.q[0]), 16);
    const uint32_t kv_lo0 = umma_desc_lo(smem_u32(sm.kv[0][0]), 16);            // as K (K-major)
    const uint32_t v_lo0 = umma_desc_lo(smem_u32(sm.kv[0][0]), kTileN * 128);   // as V (MN-major)
    constexpr uint32_t slot_step = (2 * kTileN * 64 * 2) >> 4;                  // 16 KB per ring slot
    auto issue_qk = [&](int t) -> bool {
      const int slot = (2 * t) % kSlots;
      bool got = mbar_wait(&sm.kv_full[slot], ((2 * t) / kSlots) & 1, &sm.abort_flag, p.status, 121);
      got = __all_sync(0xffffffffu, got);
      if (!got) return false;
      issue_qk64<Type>(tmem + kColS + (t & 1) * kTileN, q_lo0, kv_lo0 + slot * slot_step, &sm.done[slot]);
      return true;
    };
    bool ok = mbar_wait(&sm.q_full, 0, &sm.abort_flag, p.status, 120);
    ok = __all_sync(0xffffffffu, ok);
    ok = ok && issue_qk(0);
    for (int t = 0; ok && t < num_tiles; ++t) {
      if (t + 1 < num_tiles && !issue_qk(t + 1)) break;
      const int g = 2 * t + 1;
      const int slot = g % kSlots;
      ok = mbar_wait2(&sm.p_full[t & 1], (t >> 1) & 1, &sm.kv_full[slot], (g / kSlots) & 1, &sm.abort_flag, p.status, 122);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      issue_pv64<Type>(tO, tmem + kColS + (t & 1) * kTileN, v_lo0 + slot * slot_step, t > 0, &sm.done[slot]);
    }
  } else {
    // =============================== softmax / epilogue =================================
    const uint32_t lane_base = static_cast<uint32_t>(warp * 32) << 16;
    const float scale_log2 = p.scale_log2;
    const int row = q0 + tid;                 // in the sequence
    const bool row_valid = row < q_len;       // rows behind the sequence's end belong to others; nothing of them is kept
    const int row_keys = p.causal ? min(max(row + 1 + shift, 0), k_len) : k_len;   // keys the row sees
    // tiles that all rows of this warp see entirely (lane 0's row sees the fewest keys)
    const int warp_open = __shfl_sync(0xffffffffu, row_keys, 0) / kTileN;
    RowState st{-INFINITY, 0.f};
    bool ok = true;
    for (int t = 0; t < num_tiles; ++t) {
      const int gk = 2 * t;
      ok = mbar_wait(&sm.done[gk % kSlots], (gk / kSlots) & 1, &sm.abort_flag, p.status, 130);
      if (!(ok = __all_sync(0xffffffffu, ok))) break;
      tc_fence_after();
      const uint32_t tS = tmem + kColS + (t & 1) * kTileN + lane_base;
      uint32_t r0[32], r1[32], pk[32];
      tmem_ld32(tS, r0);
      tmem_ld32(tS + 32, r1);
      tmem_wait_ld();
      if (t >= warp_open) mask_columns_from(r0, r1, row_keys - t * kTileN);
      float2 sums = make_float2(0.f, 0.f);
      bool exact = row_valid && st.m == -INFINITY;   // nothing accumulated yet: no reference maximum to try
      if (!__any_sync(0xffffffffu, exact)) {
        sums = softmax_group_fast<Type>(r0, r1, scale_log2, st.m, pk);
        exact = row_valid && !(sums.x + sums.y <= 256.0f);   // logits outgrew the running maximum (or NaN)
      }
      if (__any_sync(0xffffffffu, exact)) {
        // Rows whose reference has to move take their own maximum of the tile; the others keep theirs and get the same P
        // again, so that a row's result does not depend on its neighbours (later tokens, with a causal mask).
        float alpha = 1.f;
        if (exact) {
          float top = -INFINITY;
#pragma unroll
          for (int j = 0; j < 32; ++j) top = fmaxf(top, fmaxf(__uint_as_float(r0[j]), __uint_as_float(r1[j])));
          top *= scale_log2;
          if (top > st.m) {
            alpha = fast_exp2(st.m - top);   // 0 when nothing was accumulated yet
            st.m = top;
            st.l *= alpha;
          }
        }
        // (a row whose logits so far are all -inf: 2^(-inf - 0) = 0, not NaN)
        sums = softmax_group_fast<Type>(r0, r1, scale_log2, st.m == -INFINITY ? 0.f : st.m, pk);
        if (t > 0) {
          // O must be quiescent: wait until P_{t-1} V_{t-1} (which read ring load 2t-1) has drained
          const int gp = 2 * t - 1;
          ok = mbar_wait(&sm.done[gp % kSlots], (gp / kSlots) & 1, &sm.abort_flag, p.status, 132);
          if (!(ok = __all_sync(0xffffffffu, ok))) break;
          tc_fence_after();
          rescale_accumulator_row(tO + lane_base, alpha);
          if (lane == 0) atomicAdd(p.slow_path_events, 1ull);
        }
      }
      st.l += sums.x + sums.y;
      tmem_st32(tS, pk);  // P_t over the first 32 columns of S_t
      tmem_wait_st();
      if (t >= open_tiles) {
        // some row of the CTA does not see all of this tile's keys
        const int g = 2 * t + 1;
        ok = mbar_wait(&sm.kv_full[g % kSlots], (g / kSlots) & 1, &sm.abort_flag, p.status, 133);
        if (!(ok = __all_sync(0xffffffffu, ok))) break;
        const int key = tid & 63;
        if (clean_half_row<Type>(sm.kv[g % kSlots][tid >> 6], key)) {
          if (t * kTileN + key < k_len) sm.special = 1;
          fence_proxy_async_smem();
        }
      }
      tc_fence_before();
      mbar_arrive(&sm.p_full[t & 1]);
    }
    // ---- epilogue: O / l -> 16 bits -> shared memory (the dead Q tile) -> global, each warp its own rows --------
    if (ok) {
      const int gl = 2 * (num_tiles - 1) + 1;   // the last P V read this load's slot
      ok = mbar_wait(&sm.done[gl % kSlots], (gl / kSlots) & 1, &sm.abort_flag, p.status, 131);
    }
    named_barrier_sync(1, kSoftmaxThreads);     // (all threads reach it; `special` is settled)
    if (*reinterpret_cast<volatile int*>(&sm.abort_flag) == 0) {
      tc_fence_after();
      // a row of no keys has accumulated P = 0: zeros
      const float inv_l = st.l > 0.f ? (1.f / st.l) : (st.l == 0.f ? 0.f : st.l);
      stage_output_half<Type>(tO + lane_base, true, inv_l, reinterpret_cast<__nv_bfloat16*>(sm.q[0]), tid);
      stage_output_half<Type>(tO + lane_base + 64, true, inv_l, reinterpret_cast<__nv_bfloat16*>(sm.q[1]), tid);
      if (*reinterpret_cast<volatile int*>(&sm.special) != 0 && row_valid) {
        // what was taken out of V in the masked tiles: a probability times an infinity or NaN is that infinity or NaN
        for (int d = 0; d < kHeadDim; d += 2) {
          uint32_t* at = reinterpret_cast<uint32_t*>(reinterpret_cast<uint8_t*>(sm.q[d >> 6]) + tid * 128 +
                                                     ((((d & 63) >> 3) ^ (tid & 7)) << 4) + (d & 7) * 2);
          float2 sum = Type::unpack(*at);
          bool any = false;
          for (int j = open_tiles * kTileN; j < row_keys; ++j) {
            const uint32_t x = __ldcg(reinterpret_cast<const uint32_t*>(static_cast<const uint16_t*>(p.v) +
                                                                        (k_rows.x + j) * p.v_stride_t + kv_head * p.v_stride_h + d));
            const uint32_t bad = non_finite_pair<Type>(x);
            const float2 f = Type::unpack(x);
            if (bad & 0x8000u) sum.x += f.x;
            if (bad & 0x80000000u) sum.y += f.y;
            any = any || bad != 0u;
          }
          if (any) *at = Type::pack(sum.x, sum.y);
        }
      }
      __syncwarp();
      // sixteen threads to a row's 256 bytes
      uint16_t* o = static_cast<uint16_t*>(p.o) + (q_rows.x + static_cast<int64_t>(q0)) * p.o_stride_t + head * p.o_stride_h;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int r = warp * 32 + 2 * i + (lane >> 4);
        const int chunk = lane & 7;
        const uint4 x = *reinterpret_cast<const uint4*>(reinterpret_cast<const uint8_t*>(sm.q[(lane >> 3) & 1]) + r * 128 +
                                                        ((chunk ^ (r & 7)) << 4));
        if (q0 + r < q_len) *reinterpret_cast<uint4*>(o + r * p.o_stride_t + (lane & 15) * 8) = x;
      }
      if (p.lse != nullptr && row_valid)
        p.lse[static_cast<int64_t>(head) * p.total_q + q_rows.x + row] = (st.m + log2f(st.l)) * 0.69314718055994531f;
    }
  }

  // ---- teardown ------------------------------------------------------------------------
  tc_fence_before();
  __syncthreads();
  if (warp == 4 && sm.abort_flag != 0) {
    // given up: the loads in flight must have landed before the CTA leaves (bounded like every wait)
    auto drain = [&](uint64_t* bar, uint32_t phase) {
      for (uint32_t n = 0; n < kSpinLimit && !mbar_try_wait(bar, phase); ++n) {
      }
    };
    for (int i = max(loads_issued - kSlots, 0); i < loads_issued; ++i) drain(&sm.kv_full[i % kSlots], (i / kSlots) & 1);
    drain(&sm.q_full, 0);
  }
  if (warp == 5) {
    __syncwarp();
    tmem_dealloc(tmem, kTmemCols);
  }
}

template <class Type>
cudaError_t launch(const CUtensorMap& tq, const CUtensorMap& tk, const CUtensorMap& tv, const PackedParams& p,
                   cudaStream_t stream) {
  auto kernel = attn_packed_kernel<Type>;
  const int smem = static_cast<int>(sizeof(PackedSmem));
  static_assert(sizeof(PackedSmem) <= 113 * 1024, "two CTAs per SM");
  static SmemLimit limit;  // per template instantiation
  cudaError_t e = ensure_dynamic_smem(kernel, smem, limit);
  if (e != cudaSuccess) return e;
  return launch_overlapped(kernel, static_cast<long long>(p.tiles) * p.heads_q, p.max_ctas, kThreads, smem, stream, tq, tk, tv, p);
}

}  // namespace

cudaError_t launch_attn_packed(const CUtensorMap& tq, const CUtensorMap& tk, const CUtensorMap& tv, const PackedParams& p,
                               bool fp16, cudaStream_t stream) {
  return fp16 ? launch<Fp16Type>(tq, tk, tv, p, stream) : launch<Bf16Type>(tq, tk, tv, p, stream);
}

}  // namespace sparsed
