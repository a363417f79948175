// Attention over packed sequences (attention_packed.cu) for long ones: the tensor-core instructions span a PAIR of CTAs on
// neighbouring SMs, as in attention_dense_pair.cu, whose pipeline this is. A cluster of two owns four consecutive tiles of up to
// 128 query rows (tokens times heads of a group) as two STREAMS of two tiles, one in each CTA; each CTA fetches half of every K and
// V tile, and both streams read it from one ring. What differs:
//   * a cluster finds its tokens in the offsets (packed_rows.cuh), and the streams walk up to their own last tokens' keys; a
//     slot that only the second stream still reads is free when that has read it
//   * masked tiles, the last ones of a walk. V's infinities and NaN are taken out there as in attention_packed.cu, by the softmax
//     warps of each CTA in the half that it holds. So a CTA has to know that its own half has landed: those loads count on the
//     CTA's own barrier instead of the leader's. That the peer's half is there and clean, the leader's issuer knows from the
//     peer's softmax warps, which hand over P only then. (A CTA's barrier serves each masked tile with a slot of its own: at
//     most ten tiles of 64 keys can be masked for 512 tokens, and the ring has ten slots for V.)
//   * rows go out from the staged tile with ordinary stores: the tile at a sequence's end must not touch the next sequence.
// When a call comes here: packed_pair_pays (dense_choice.h). Roundings as there. Bound by the power limit: 32768 tokens x 32 heads,
// causal, 8.8 T operations in 7.0 to 7.1 ms (1.24 PFLOP/s; the single-CTA kernel 7.5), 2 x 8192 x 32 heads without a mask 1.81 ms
// (1.21; 1.97).
#include <type_traits>

#include "internal.h"
#include "packed_rows.cuh"
#include "sm100_pair_primitives.cuh"

namespace sparsed {
namespace {

constexpr int kHeadDim = 128;
constexpr int kTileM = 128;        // query rows per CTA and stream
constexpr int kTileN = 64;         // keys per pipeline step
constexpr int kStreams = 2;
constexpr int kSlots = 20;         // 8 KB ring slots (half a K tile or half a V tile each), shared by both streams
constexpr int kThreads = 384;      // warps 0-3 / 4-7: softmax of stream 0 / 1; 8: producer; 10, 11: issuers
constexpr int kTmemCols = 512;     // per stream 256: two S buffers of 64 columns, then O (128)
constexpr int kColS = 0;
constexpr int kColO = 128;
constexpr int kArrivalsP = 8;      // four softmax warps in each CTA of the pair

struct PairStream {
  alignas(1024) uint16_t q[2][kTileM * 64];           // two 64-wide halves of head_dim; stages the output too
  uint64_t q_full;                    // used in the leader CTA: bytes of both CTAs
  uint64_t done[kSlots];              // in both CTAs: this stream's MMAs that read the slot have completed
  uint64_t p_full[2];                 // used in the leader CTA: P of both CTAs is in tensor memory
};

struct PairSmem {
  // K half-tile: two [32 keys x 64] halves of head_dim (4 KB each); V half-tile: [64 keys x 64 columns of head_dim].
  alignas(1024) uint16_t kv[kSlots][kTileN * 64];
  PairStream stream[kStreams];
  uint64_t kv_full[kSlots];           // in the leader CTA: bytes of both CTAs; V of masked tiles: this CTA's bytes, in each CTA
  uint32_t tmem_base;
  int abort_flag;
  int special;                        // in both CTAs: a V of the sequence in a masked tile is infinite or NaN
};

constexpr uint32_t kHi = umma_desc_hi_sw128(1024);
constexpr uint32_t kIdescQK = umma_idesc_bf16(256, 64, false, false);    // S = Q K^T, both K-major
constexpr uint32_t kIdescPV = umma_idesc_bf16(256, 128, false, true);    // O += P V, V MN-major
constexpr uint32_t kQHalfStep = (kTileM * 64 * 2) >> 4;                  // 16 KB per head_dim half of Q
constexpr uint32_t kKHalfStep = (32 * 64 * 2) >> 4;                      // 4 KB per head_dim half of a K half-tile
constexpr uint32_t kSlotStep = (kTileN * 64 * 2) >> 4;                   // 8 KB per ring slot

template <class Type>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
attn_packed_pair_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                        const __grid_constant__ CUtensorMap tm_v, const PackedParams p) {
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  PairSmem& sm = *reinterpret_cast<PairSmem*>(smem_raw);
  const int tid = threadIdx.x;
  const int warp = tid >> 5;
  const int lane = tid & 31;
  const int rank = static_cast<int>(cluster_cta_rank());   // 0 = leader
  // (both CTAs of a pair take this exit, or the next one, or neither)
  if ((smem_u32(smem_raw) & 1023u) != 0u) {
    if (tid == 0) record_status(p.status, 2, 6);
    return;
  }
  // ---- which rows ---------------------------------------------------------------------------
  const int2 tile_head = packed_tile_and_head(p, blockIdx.x >> 1);
  PackedTokens it;
  if (!packed_tokens(p, tile_head.x, 4 * p.tile_tokens, it)) return;   // an empty tile
  const int head = tile_head.y * p.pack, kv_head = head / p.group, group_head = head - kv_head * p.group;
  // Stream s of CTA r has tokens [(2 s + r) * tile_tokens, + tile_tokens); a stream without any has no rows at all, one whose
  // peer tile has none still runs as a pair: the peer's rows are nobody's.
  const int T = p.tile_tokens;
  // tiles all of whose keys all rows of the cluster see, an even number
  const int open_tiles = it.keys_of(0, p.causal) / kTileN & ~1;
  auto stream_tiles = [&](int s) -> int {
    if (2 * s * T >= it.tokens) return 0;
    return (it.keys_of(min((2 * s + 2) * T, it.tokens) - 1, p.causal) + kTileN - 1) / kTileN;
  };
  const int tiles0 = stream_tiles(0), tiles1 = stream_tiles(1), all_tiles = max(tiles0, tiles1);

  // ---- set-up -------------------------------------------------------------------------------
  if (tid == 0) {
    for (int s = 0; s < kStreams; ++s) {
      PairStream& S = sm.stream[s];
      mbar_init(&S.q_full, 1);
      for (int i = 0; i < kSlots; ++i) mbar_init(&S.done[i], 1);
      mbar_init(&S.p_full[0], kArrivalsP);
      mbar_init(&S.p_full[1], kArrivalsP);
    }
    for (int i = 0; i < kSlots; ++i) mbar_init(&sm.kv_full[i], 1);
    sm.abort_flag = 0;
    sm.special = 0;
    mbar_fence_init();
  }
  if (warp == 8 && elect_one_sync()) {
    tma_prefetch_desc(&tm_q);
    tma_prefetch_desc(&tm_k);
    tma_prefetch_desc(&tm_v);
  }
  if (warp == 10) {
    tmem_alloc_pair(&sm.tmem_base, kTmemCols);
    tmem_relinquish_pair();
  }
  tc_fence_before();
  __syncthreads();
  // the peer's barriers must exist before anything is signalled on them
  cluster_arrive();
  cluster_wait();
  tc_fence_after();
  const uint32_t tmem = sm.tmem_base;
  bool pair_ok = true;
  {
    // the pair's instructions address both tensor memories with one base: never expected to differ
    const uint32_t peer_base = ld_cluster_u32(map_to_cta(smem_u32(&sm.tmem_base), rank ^ 1u));
    if (peer_base != tmem) {
      pair_ok = false;
      if (tid == 0) record_status(p.status, 4, 2);
    }
  }

  const int s_of_warp = warp < 8 ? (warp >> 2) : ((warp - 8) & 1);   // stream this warp serves
  PairStream& S = sm.stream[s_of_warp];
  const int num_tiles = s_of_warp == 0 ? tiles0 : tiles1;
  const uint32_t tS0 = tmem + s_of_warp * 256 + kColS;
  const uint32_t tO = tmem + s_of_warp * 256 + kColO;
  const bool has_rows = 2 * s_of_warp * T < it.tokens;

  if (!pair_ok || !has_rows) {
    // nothing to do for this warp
  } else if (warp == 9) {
    // (spare warp)
  } else if (warp == 8) {
    // =============================== TMA producer (both streams) =============================
    bool ok = true;
    for (int s = 0; s < kStreams; ++s) {
      if ((s == 0 ? tiles0 : tiles1) > 0 && elect_one_sync()) {
        PairStream& X = sm.stream[s];
        const uint32_t q_full_leader = map_to_cta(smem_u32(&X.q_full), 0);
        const int row0 = it.q_row + (2 * s + rank) * T;   // (rows beyond the tensor arrive as zeros)
        if (rank == 0) mbar_expect_tx(&X.q_full, 2 * T * p.pack * kHeadDim * 2);
        tma_load_4d_pair(X.q[0], &tm_q, q_full_leader, 0, group_head, row0, kv_head);
        tma_load_4d_pair(X.q[1], &tm_q, q_full_leader, 64, group_head, row0, kv_head);
      }
      __syncwarp();
    }
    // load i: this CTA's half of K (even) or V (odd) of tile i / 2, for both streams
    int issued = 0;
    for (int i = 0; i < 2 * all_tiles; ++i) {
      const int slot = i % kSlots, t = i >> 1;
      if (i >= kSlots) {
        // free once the MMAs of every stream that read it have completed
        const uint32_t parity = ((i / kSlots) - 1) & 1;
        const int before = (i - kSlots) >> 1;   // the tile that was there
        uint64_t* done0 = &sm.stream[0].done[slot];
        uint64_t* done1 = &sm.stream[1].done[slot];
        ok = before < min(tiles0, tiles1) ? mbar_wait2(done0, parity, done1, parity, &sm.abort_flag, p.status, 140)
                                          : mbar_wait(before < tiles1 ? done1 : done0, parity, &sm.abort_flag, p.status, 140);
        if (!(ok = __all_sync(0xffffffffu, ok))) break;
      }
      if (elect_one_sync()) {
        const int key0 = it.k_row + t * kTileN;
        if ((i & 1) == 0) {
          // keys [32 rank, 32 rank + 32) of the tile, all of head_dim
          const uint32_t full_leader = map_to_cta(smem_u32(&sm.kv_full[slot]), 0);
          if (rank == 0) mbar_expect_tx(&sm.kv_full[slot], 2 * kTileN * 64 * 2);   // both CTAs' halves
          tma_load_4d_pair(sm.kv[slot], &tm_k, full_leader, 0, key0 + 32 * rank, kv_head, 0);
          tma_load_4d_pair(sm.kv[slot] + 32 * 64, &tm_k, full_leader, 64, key0 + 32 * rank, kv_head, 0);
        } else {
          // all 64 keys, head_dim columns [64 rank, 64 rank + 64)
          const bool masked = t >= open_tiles;
          if (rank == 0 || masked) mbar_expect_tx(&sm.kv_full[slot], (masked ? 1 : 2) * kTileN * 64 * 2);
          tma_load_4d_pair(sm.kv[slot], &tm_v, map_to_cta(smem_u32(&sm.kv_full[slot]), masked ? rank : 0), 64 * rank, key0, kv_head, 0);
        }
      }
      __syncwarp();
      issued = i + 1;
    }
    // given up: what this CTA's barriers count must land before the cluster leaves (bounded like every wait)
    for (int i = max(issued - kSlots, 0); !ok && i < issued; ++i) {
      const bool own = (i & 1) != 0 && (i >> 1) >= open_tiles;
      if (rank != 0 && !own) continue;
      for (uint32_t n = 0; n < kSpinLimit && !mbar_try_wait(&sm.kv_full[i % kSlots], rank == 0 ? (i / kSlots) & 1 : 0); ++n) {
      }
    }
  } else if (warp == 10 || warp == 11) {
    // =============================== UMMA issuer (leader CTA) ================================
    if (rank == 0 && num_tiles > 0) {
      const uint32_t q_lo0 = umma_desc_lo(smem_u32(S.q[0]), 16);
      const uint32_t k_lo0 = umma_desc_lo(smem_u32(sm.kv[0]), 16);             // as K (K-major)
      const uint32_t v_lo0 = umma_desc_lo(smem_u32(sm.kv[0]), kTileN * 128);   // as V (MN-major, one 64-wide atom)
      // S_t = Q K_t^T into S buffer t & 1: eight M256 N64 K16 MMAs
      auto issue_qk = [&](int t) -> bool {
        const int g = 2 * t;
        const int slot = g % kSlots;
        bool got = mbar_wait(&sm.kv_full[slot], (g / kSlots) & 1, &sm.abort_flag, p.status, 141);
        got = __all_sync(0xffffffffu, got);
        if (!got) return false;
        tc_fence_after();
        if (elect_one_sync()) {
          const uint32_t d = tS0 + (t & 1) * kTileN;
          const uint32_t k_lo = k_lo0 + slot * kSlotStep;
          umma_ss_pair<false>(d, q_lo0, kHi, k_lo, kHi, Type::idesc(kIdescQK));
#pragma unroll
          for (int kk = 1; kk < 8; ++kk)
            umma_ss_pair<true>(d, q_lo0 + (kk >> 2) * kQHalfStep + (kk & 3) * 2, kHi,
                               k_lo + (kk >> 2) * kKHalfStep + (kk & 3) * 2, kHi, Type::idesc(kIdescQK));
          umma_commit_pair(&S.done[slot]);
        }
        __syncwarp();
        return true;
      };
      bool ok = mbar_wait(&S.q_full, 0, &sm.abort_flag, p.status, 142);
      ok = __all_sync(0xffffffffu, ok);
      ok = ok && issue_qk(0);
      for (int t = 0; ok && t < num_tiles; ++t) {
        // The S buffer of tile t+1 last held P of tile t-1, whose P V was issued earlier by this thread, and
        // tcgen05 operations of one thread execute in issue order.
        if (t + 1 < num_tiles && !(ok = issue_qk(t + 1))) break;
        const int g = 2 * t + 1;
        const int slot = g % kSlots;
        ok = mbar_wait2(&S.p_full[t & 1], (t >> 1) & 1, &sm.kv_full[slot], (g / kSlots) & 1, &sm.abort_flag, p.status, 143);
        if (!(ok = __all_sync(0xffffffffu, ok))) break;
        tc_fence_after();
        if (elect_one_sync()) {
          // O (+)= P_t V_t: four M256 N128 K16 MMAs, 16 keys (2048 bytes of V) per step
          const uint32_t a = tS0 + (t & 1) * kTileN;
          const uint32_t v_lo = v_lo0 + slot * kSlotStep;
          umma_ts_pair(tO, a, v_lo, kHi, Type::idesc(kIdescPV), t > 0 ? 1u : 0u);
#pragma unroll
          for (int kk = 1; kk < 4; ++kk) umma_ts_pair(tO, a + kk * 8, v_lo + kk * 128, kHi, Type::idesc(kIdescPV), 1u);
          umma_commit_pair(&S.done[slot]);
        }
        __syncwarp();
      }
    }
  } else {
    // =============================== softmax / epilogue ======================================
    const int row = tid & (kTileM - 1);   // in the tile
    const uint32_t lane_base = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const float scale_log2 = p.scale_log2;
    const int token = row / p.pack;       // of the tile's
    const int my_token = (2 * s_of_warp + rank) * T + token;
    const bool row_valid = token < T && my_token < it.tokens;   // (rows behind the sequence's end are nobody's)
    auto row_keys = [&]() -> int { return it.keys_of(my_token, p.causal); };
    const uint32_t p_full_leader0 = map_to_cta(smem_u32(&S.p_full[0]), 0);
    const uint32_t p_full_leader1 = map_to_cta(smem_u32(&S.p_full[1]), 0);
    bool ok = true;
    // (a row that is nobody's holds anything: a finite reference keeps it from asking for the exact path in every tile)
    RowState st{row_valid ? -INFINITY : 0.f, 0.f};
    // One tile. kind: 0 / 1 = seen entirely by all rows, even / odd (compile-time, as its S buffer then is); 2 = masked.
    auto tile_body = [&](int t, auto kind) -> bool {
      constexpr int kKind = decltype(kind)::value;
      bool got;
      if constexpr (kKind == 2) {
        // Some row of the cluster does not see all of these keys: this CTA's half of V is looked at while S_t is still being
        // worked out, by the warps of both streams (whichever comes first finds something, and says so to all of the cluster).
        const int slot = (2 * t + 1) % kSlots;
        const uint32_t phase = rank == 0 ? ((2 * t + 1) / kSlots) & 1 : 0;   // (the peer's barrier serves masked tiles alone)
        got = mbar_wait(&sm.kv_full[slot], phase, &sm.abort_flag, p.status, 147);
        if (!__all_sync(0xffffffffu, got)) return false;
        const int key = row & 63;
        if (row < 64) {
          if (has_non_finite<Type>(sm.kv[slot], key)) {
            if (t * kTileN + key < it.k_len) {
              *reinterpret_cast<volatile int*>(&sm.special) = 1;
              st_cluster_u32(map_to_cta(smem_u32(&sm.special), rank ^ 1u), 1u);
            }
            asm volatile("fence.acq_rel.cluster;" ::: "memory");
            clean_half_row<Type>(sm.kv[slot], key);
          }
          // Also where nothing was found: the other stream's thread may just have cleaned the row and not be here yet. The zeros
          // that this thread has read then come before this stream's MMA, and with the last tile the other's note before this
          // stream's epilogue in either CTA. (The wider fence in every masked tile: 1 % of a causal 32k prompt.)
          if (t + 1 == num_tiles) asm volatile("fence.acq_rel.cluster;" ::: "memory");
          fence_proxy_async_smem();
        }
      }
      // S_t is ready when the Q K^T batch that read ring load 2t has completed
      const int gk = 2 * t;
      got = mbar_wait(&S.done[gk % kSlots], (gk / kSlots) & 1, &sm.abort_flag, p.status, 144);
      if (!__all_sync(0xffffffffu, got)) return false;
      tc_fence_after();
      const int buf = kKind == 2 ? t & 1 : kKind;
      const uint32_t tS = tS0 + buf * kTileN + lane_base;
      uint32_t r0[32], r1[32], pk[32];
      tmem_ld32(tS, r0);
      tmem_ld32(tS + 32, r1);
      tmem_wait_ld();
      if constexpr (kKind == 2) {
        const int valid = row_keys() - t * kTileN;
        const int least = __reduce_min_sync(0xffffffffu, valid);
        if (least < 32) mask_half(r0, valid);
        if (least < 64) mask_half(r1, valid - 32);
      }
      float2 sums = make_float2(0.f, 0.f);
      bool exact = st.m == -INFINITY;   // nothing accumulated yet: no reference maximum to try
      if (!__any_sync(0xffffffffu, exact)) {
        sums = softmax_group_fast<Type>(r0, r1, scale_log2, st.m, pk);
        exact = sums.x + sums.y > Type::kMostSum;
      }
      if (__any_sync(0xffffffffu, exact)) {
        // (as in attention_packed.cu)
        float alpha = 1.f;
        if (exact) {
          float top = -INFINITY;
#pragma unroll
          for (int j = 0; j < 32; ++j) top = fmaxf(top, fmaxf(__uint_as_float(r0[j]), __uint_as_float(r1[j])));
          top = top * scale_log2 - Type::kHeadroom;
          if (top > st.m) {
            alpha = fast_exp2(st.m - top);   // 0 when nothing was accumulated yet
            st.m = top;
            st.l *= alpha;
          }
        }
        sums = softmax_group_fast<Type>(r0, r1, scale_log2, st.m == -INFINITY ? 0.f : st.m, pk);
        if (t > 0) {
          // O must be quiescent: wait until P_{t-1} V_{t-1} (which read ring load 2t-1) has drained
          const int gp = 2 * t - 1;
          got = mbar_wait(&S.done[gp % kSlots], (gp / kSlots) & 1, &sm.abort_flag, p.status, 145);
          if (!__all_sync(0xffffffffu, got)) return false;
          tc_fence_after();
          rescale_accumulator_row(tO + lane_base, alpha);
          if (lane == 0) atomicAdd(p.slow_path_events, 1ull);
        }
      }
      st.l += sums.x + sums.y;
      tmem_st32(tS, pk);  // P_t over the first 32 columns of S_t
      tmem_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive_cluster(buf ? p_full_leader1 : p_full_leader0);
      return true;
    };
    {
      int t = 0;
      const int open = min(open_tiles, num_tiles & ~1);
      for (; ok && t < open; t += 2)
        ok = tile_body(t, std::integral_constant<int, 0>{}) && tile_body(t + 1, std::integral_constant<int, 1>{});
      for (; ok && t < num_tiles; ++t) ok = tile_body(t, std::integral_constant<int, 2>{});
    }
    // ---- epilogue: O / l -> 16 bits -> shared memory (the dead Q tile) -> global, each warp its own rows ----------
    if (ok && num_tiles > 0) {
      const int gl = 2 * num_tiles - 1;   // the last P V read this load's slot
      ok = mbar_wait(&S.done[gl % kSlots], (gl / kSlots) & 1, &sm.abort_flag, p.status, 146);
    }
    if (__all_sync(0xffffffffu, ok)) {
      tc_fence_after();
      const float inv_l = st.l > 0.f ? (1.f / st.l) : (st.l == 0.f ? 0.f : st.l);   // (a row of no keys: zeros)
      stage_output_half<Type>(tO + lane_base, num_tiles > 0, inv_l, reinterpret_cast<__nv_bfloat16*>(S.q[0]), row);
      stage_output_half<Type>(tO + lane_base + 64, num_tiles > 0, inv_l, reinterpret_cast<__nv_bfloat16*>(S.q[1]), row);
      if (*reinterpret_cast<volatile int*>(&sm.special) != 0 && row_valid)
        add_special<Type>(p, S.q, row, it.k_row, open_tiles * kTileN, row_keys(), kv_head);
      __syncwarp();
      uint4 x[16];
      read_staged_rows(S.q, row & ~31, lane, x);
      const int q_row = it.q_row + my_token, q_head = head + row - token * p.pack;
      store_rows(p.o, row_valid ? static_cast<int64_t>(q_row) * p.o_stride_t + q_head * p.o_stride_h : -1, lane, x);
      if (p.lse != nullptr && row_valid)
        p.lse[static_cast<int64_t>(q_head) * p.total_q + q_row] = st.l == 0.f ? -INFINITY : (st.m + log2f(st.l)) * 0.69314718055994531f;
    }
  }

  // ---- teardown -------------------------------------------------------------------------------
  // neither CTA may leave (or free its tensor memory) while the pair's MMAs, loads or arrivals can still touch it
  tc_fence_before();
  __syncthreads();
  cluster_arrive();
  cluster_wait();
  if (warp == 10) {
    __syncwarp();
    tmem_dealloc_pair(tmem, kTmemCols);
  }
}

template <class Type>
cudaError_t launch_pair(const CUtensorMap& tq, const CUtensorMap& tk, const CUtensorMap& tv, const PackedParams& p,
                        cudaStream_t stream) {
  auto kernel = attn_packed_pair_kernel<Type>;
  const int smem = static_cast<int>(sizeof(PairSmem));
  static_assert(sizeof(PairSmem) <= 227 * 1024, "one CTA per SM");
  static SmemLimit limit;  // per template instantiation
  cudaError_t e = ensure_dynamic_smem(kernel, smem, limit);
  if (e != cudaSuccess) return e;
  return launch_overlapped(kernel, 2ll * p.tiles * (p.heads_q / p.pack), 0, kThreads, smem, stream, tq, tk, tv, p);
}

}  // namespace

// K's tensor map: boxes of 64 x 32 rows. p.tiles counts tiles of 4 * p.tile_tokens tokens.
cudaError_t launch_attn_packed_pair(const CUtensorMap& tq, const CUtensorMap& tk, const CUtensorMap& tv, const PackedParams& p,
                                    bool fp16, cudaStream_t stream) {
  return fp16 ? launch_pair<Fp16Type>(tq, tk, tv, p, stream) : launch_pair<Bf16Type>(tq, tk, tv, p, stream);
}

}  // namespace sparsed
