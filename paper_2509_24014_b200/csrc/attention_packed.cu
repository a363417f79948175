// Attention over packed sequences of different lengths, causal or not, head_dim 128, bf16 or fp16, fp32 softmax, on sm_100a.
//
// An item is a tile of up to 128 query rows that share their keys: some consecutive tokens of one sequence times some query
// heads of one key-value head (grouped heads: a tile of 18 tokens x 7 heads is full where 128 tokens of one head are not there,
// and the diagonal of a causal mask cuts through fewer of its keys). It runs the pipeline of attention.cu over the sequence's
// keys, 64 at a time, up to the last one that its last token sees: a producer warp (TMA into a ring of swizzled tiles), a warp
// that issues S_t = Q K_t^T and O += P_t V_t with S, P and O in tensor memory, and four warps with a thread per query row
// (softmax_pipeline.cuh). Two CTAs per SM.
//
// CTAs run from one item into the next, each role by itself: a CTA takes over CTAs of the grid that have not been launched yet
// (cluster launch control, as the packed walks of attention.cu), and its producer finds the next item's rows and sends its
// first loads off while the softmax warps are still in the one before. So only a CTA's first item pays for the chain from the
// offsets over the first loads to the first softmax, and items of different lengths are balanced.
//
// Which rows: the lengths are only known on the device. With tiles of T tokens, sequence b gets the tile numbers from
// cu_q[b] / T + b on: that leaves it room for at least ceil(len / T) tiles, ascends with b, and needs no sum over the sequences
// before it, so an item's sequence is found by one search in cu_q, and the number of tiles, total_q / T + num_seqs, is known
// to the host. Numbers beyond a sequence's last tile are empty and passed over (at most one for each sequence).
//
// What a row must not see: with a causal mask the logits beyond each row's last key are set to -inf, in the tiles that the
// diagonal or the sequence's end runs through; all other tiles are walked without a comparison. P is then 0 there, but 0 * V is
// not 0 for a V that is infinite or NaN, and the tile at a sequence's end holds rows of the next sequence, or rows that nobody
// has written yet. So in those tiles the softmax threads look at V in shared memory before they hand P over: what is not
// finite becomes 0 there, and where it belongs to a key of this sequence, which some rows of the tile see, it is added to
// those rows' outputs in the epilogue, element by element.
//
// Roundings: logits, softmax sums and O are fp32. P goes to the tensor cores in the inputs' 16-bit type, which the MMA wants for both
// operands: up to half a step of it per weight (2^-8 of the weight in bf16, 2^-11 in fp16), with either sign, while the sum takes
// it unrounded; O is rounded once, at the end. Errors against 64 bits, of O's size: bf16 2.2e-3, fp16 2.9e-4, where rounding an
// exact O alone gives 1.7e-3 and 2.1e-4.
//
// Bound: as the dense kernel, the tensor pipe and the softmax warps at the power limit (the device draws 1000 W and runs at
// 1.36 GHz in such calls); a launch by itself, with the clock at its highest, takes 0.88 of that time with tensor pipe and
// exponential unit busy 60 to 63 % each, the rest being the latency of a tile's steps and of the first and last items; short
// sequences by what an item costs beside its tiles, about three tiles' worth. Measured, on visible (row, key) pairs: 12 prompts
// of 165 to 3321 tokens, 28 heads on 4, some with cached text, causal, 0.79 T operations in 790 us (1.0 PFLOP/s); 8 sequences
// of 512 to 3980 tokens x 32 heads, no mask, fp16, 0.84 T in 885 to 917 us (0.93); six turns of 1 to 160 tokens x 8 heads, 8.5
// us in a graph. In-order taking of items leaves 2.5 % of either batch's time to its last items.
// Not kept: four or six ring slots (2 % slower; no room), the next item fetched earlier (2 %), loads sent off before the barriers
// are set up (short calls 0.2 us faster, 512 tokens 5 % slower), rows stored from tensor memory without the staging (7 %), a loop
// of two open tiles (spills, 10 %).
#include "packed_rows.cuh"
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

// What the roles of a CTA need to know of an item.
struct PackedItem : PackedTokens {
  int num_tiles;     // 64-key tiles to walk; -1: no more items
  int open_tiles;    // the first of them, all of whose keys all rows see
  int head;          // first query head
};

struct PackedSmem {
  alignas(1024) uint16_t q[2][kTileM * 64];           // two 64-wide halves of head_dim; stages the output too
  alignas(1024) uint16_t kv[kSlots][2][kTileN * 64];
  uint64_t q_full, kv_full[kSlots];
  uint64_t done[kSlots];   // the MMAs that read the slot have completed
  uint64_t p_full[2];
  uint64_t q_free;         // every softmax warp has read its rows of the output out of the Q buffer: the next Q may land
  uint64_t item_full[2], item_free[2];   // the producer hands items over through two buffers
  PackedItem item[2];
  alignas(16) uint32_t control[4];       // (the launch control's answer)
  uint64_t control_full;
  uint32_t tmem_base;
  int abort_flag;
  int special[2];          // number of the item in whose masked tiles a V of its sequence is infinite or NaN
};

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

  // ---- set-up --------------------------------------------------------------------------
  if (tid == 0) {
    mbar_init(&sm.q_full, 1);
    mbar_init(&sm.q_free, 4);
    for (int s = 0; s < kSlots; ++s) {
      mbar_init(&sm.kv_full[s], 1);
      mbar_init(&sm.done[s], 1);
    }
    for (int s = 0; s < 2; ++s) {
      mbar_init(&sm.p_full[s], kSoftmaxThreads);
      mbar_init(&sm.item_full[s], 1);
      mbar_init(&sm.item_free[s], 5);   // four softmax warps and the issuer
      sm.special[s] = -1;
    }
    mbar_init(&sm.control_full, 1);
    sm.abort_flag = 0;
    mbar_fence_init();
  }
  if (warp == 5) {
    tmem_alloc(&sm.tmem_base, kTmemCols);
    tmem_relinquish();
  }
  if (warp == 4 && elect_one_sync()) {
    tma_prefetch_desc(&tm_q);
    tma_prefetch_desc(&tm_k);
    tma_prefetch_desc(&tm_v);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sm.tmem_base;
  const uint32_t tO = tmem + kColO;

  // Warps 4 and 5 run their loops with all 32 lanes converged and let one elected lane issue.
  if (warp == 4) {
    // =============================== producer ===========================================
    PackedItem it;
    // what grid number `number` is; false: an empty tile
    auto describe = [&](int number) -> bool {
      const int2 tile_head = packed_tile_and_head(p, number);
      if (!packed_tokens(p, tile_head.x, p.tile_tokens, it)) return false;
      it.head = tile_head.y * p.pack;
      it.num_tiles = (it.keys_of(it.tokens - 1, p.causal) + kTileN - 1) / kTileN;
      it.open_tiles = it.keys_of(0, p.causal) / kTileN;
      return true;
    };
    auto request_item = [&]() {
      if (elect_one_sync()) {
        mbar_expect_tx(&sm.control_full, 16);
        launch_control_request(sm.control, &sm.control_full);
      }
      __syncwarp();
    };
    auto publish = [&](int buf) {
      __syncwarp();
      if (lane == 0) {
        sm.item[buf] = it;
        mbar_arrive(&sm.item_full[buf]);
      }
      __syncwarp();
    };
    bool ok = true, asked = false;
    uint32_t requests = 0, answers = 0;   // of the launch control
    int load0 = 0, q_tiles = 0;           // K / V loads and Q tiles of earlier items
    int issued = 0, q_issued = 0;
    int number = blockIdx.x;
    for (int nth = 0; ok; ++nth) {        // the CTA's nth item, in item buffer nth & 1
      bool found = nth == 0 && describe(number);
      while (!found) {
        if (!asked) {
          request_item();
          ++requests;
        }
        asked = false;
        ok = mbar_wait(&sm.control_full, answers & 1, &sm.abort_flag, p.status, 113);
        if (!(ok = __all_sync(0xffffffffu, ok))) break;
        ++answers;
        number = launch_control_answer(sm.control);
        __syncwarp();
        if (number < 0) break;
        found = describe(number);
      }
      // the other roles have finished with the item that was in this buffer
      if (ok && nth >= 2) {
        ok = mbar_wait(&sm.item_free[nth & 1], ((nth >> 1) - 1) & 1, &sm.abort_flag, p.status, 112);
        ok = __all_sync(0xffffffffu, ok);
      }
      if (!ok) break;
      if (!found) {
        it.num_tiles = -1;
        publish(nth & 1);
        break;
      }
      publish(nth & 1);
      const int loads = 2 * it.num_tiles;
      // The Q buffer doubles as the staging tile of the output before: the next Q may land once that has been read out. The
      // first ring-full of the item's K / V loads does not depend on it and goes out first.
      bool q_pending = loads > 0;
      auto settle_q = [&]() -> bool {
        bool got = true;
        if (q_tiles > 0) {
          got = mbar_wait(&sm.q_free, (q_tiles - 1) & 1, &sm.abort_flag, p.status, 111);
          got = __all_sync(0xffffffffu, got);
        }
        if (got && elect_one_sync()) {
          mbar_expect_tx(&sm.q_full, p.tile_tokens * p.pack * kHeadDim * 2);   // rows beyond the tensor arrive as zeros
          const int group = it.head / p.group, first = it.head - group * p.group;
          tma_load_4d(sm.q[0], &tm_q, &sm.q_full, 0, first, it.q_row, group);
          tma_load_4d(sm.q[1], &tm_q, &sm.q_full, 64, first, it.q_row, group);
        }
        __syncwarp();
        if (got) ++q_issued;
        q_pending = false;
        return got;
      };
      const int kv_head = it.head / p.group;
      const int q_at = nth == 0 ? 0 : min(loads, kSlots);
      // The next item is asked for two tiles before this one's last load: late enough that a CTA with a long item does not hold
      // one that another could have started, early enough for the answer to be there.
      const int request_at = max(loads - 4, 0);
      for (int i = 0; i < loads; ++i) {
        if (q_pending && i == q_at && !(ok = settle_q())) break;
        if (i == request_at) {
          request_item();
          ++requests;
          asked = true;
        }
        const int g = load0 + i, slot = g % kSlots;
        if (g >= kSlots) {
          ok = mbar_wait(&sm.done[slot], ((g / kSlots) - 1) & 1, &sm.abort_flag, p.status, 110);
          if (!(ok = __all_sync(0xffffffffu, ok))) break;
        }
        if (elect_one_sync()) {
          const CUtensorMap* tm = (i & 1) == 0 ? &tm_k : &tm_v;
          mbar_expect_tx(&sm.kv_full[slot], kTileN * kHeadDim * 2);
          tma_load_4d(sm.kv[slot][0], tm, &sm.kv_full[slot], 0, it.k_row + (i >> 1) * kTileN, kv_head, 0);
          tma_load_4d(sm.kv[slot][1], tm, &sm.kv_full[slot], 64, it.k_row + (i >> 1) * kTileN, kv_head, 0);
        }
        __syncwarp();
        issued = g + 1;
      }
      if (ok && q_pending) ok = settle_q();
      load0 += loads;
      if (loads > 0) ++q_tiles;
    }
    if (!ok) {
      // given up: what is on its way must land before the CTA leaves (bounded like every wait)
      auto drain = [&](uint64_t* bar, uint32_t phase) {
        for (uint32_t n = 0; n < kSpinLimit && !mbar_try_wait(bar, phase); ++n) {
        }
      };
      if (requests > answers) drain(&sm.control_full, answers & 1);
      for (int g = max(issued - kSlots, 0); g < issued; ++g) drain(&sm.kv_full[g % kSlots], (g / kSlots) & 1);
      if (q_issued > 0) drain(&sm.q_full, (q_issued - 1) & 1);
    }
  } else if (warp == 5) {
    // =============================== UMMA issuer ========================================
    const uint32_t q_lo0 = umma_desc_lo(smem_u32(sm.q[0]), 16);
    const uint32_t kv_lo0 = umma_desc_lo(smem_u32(sm.kv[0][0]), 16);            // as K (K-major)
    const uint32_t v_lo0 = umma_desc_lo(smem_u32(sm.kv[0][0]), kTileN * 128);   // as V (MN-major)
    constexpr uint32_t slot_step = (2 * kTileN * 64 * 2) >> 4;                  // 16 KB per ring slot
    bool ok = true;
    int load0 = 0, tile0 = 0, q_tiles = 0;   // loads / tiles / Q tiles of earlier items
    for (int nth = 0; ok; ++nth) {
      const int buf = nth & 1;
      ok = mbar_wait(&sm.item_full[buf], (nth >> 1) & 1, &sm.abort_flag, p.status, 123);
      if (!(ok = __all_sync(0xffffffffu, ok))) break;
      const int num_tiles = sm.item[buf].num_tiles;
      __syncwarp();
      if (lane == 0) mbar_arrive(&sm.item_free[buf]);
      if (num_tiles < 0) break;
      if (num_tiles == 0) continue;
      auto issue_qk = [&](int t) -> bool {
        const int g = load0 + 2 * t, slot = g % kSlots;
        bool got = mbar_wait(&sm.kv_full[slot], (g / kSlots) & 1, &sm.abort_flag, p.status, 121);
        got = __all_sync(0xffffffffu, got);
        if (!got) return false;
        issue_qk64<Type>(tmem + kColS + ((tile0 + t) & 1) * kTileN, q_lo0, kv_lo0 + slot * slot_step, &sm.done[slot]);
        return true;
      };
      ok = mbar_wait(&sm.q_full, q_tiles & 1, &sm.abort_flag, p.status, 120);
      ok = __all_sync(0xffffffffu, ok);
      ++q_tiles;
      ok = ok && issue_qk(0);
      for (int t = 0; ok && t < num_tiles; ++t) {
        // The S buffer of tile t+1 last held P of the tile two before it, whose P V was issued
        // earlier by this thread, and tcgen05 operations of one thread execute in issue order.
        if (t + 1 < num_tiles && !(ok = issue_qk(t + 1))) break;
        const int g = load0 + 2 * t + 1, slot = g % kSlots, gt = tile0 + t;
        ok = mbar_wait2(&sm.p_full[gt & 1], (gt >> 1) & 1, &sm.kv_full[slot], (g / kSlots) & 1, &sm.abort_flag, p.status, 122);
        if (!(ok = __all_sync(0xffffffffu, ok))) break;
        // the first P V of an item overwrites O: the softmax warps handed P over after they had read the previous item's O
        issue_pv64<Type>(tO, tmem + kColS + (gt & 1) * kTileN, v_lo0 + slot * slot_step, t > 0, &sm.done[slot]);
      }
      load0 += 2 * num_tiles;
      tile0 += num_tiles;
    }
  } else {
    // =============================== softmax / epilogue =================================
    const uint32_t lane_base = static_cast<uint32_t>(warp * 32) << 16;
    const float scale_log2 = p.scale_log2;
    const int token = tid / p.pack;   // this thread's row of every item: this token, head tid % pack
    bool ok = true;
    int load0 = 0, tile0 = 0;   // loads / tiles of earlier items
    for (int nth = 0; ok; ++nth) {
      ok = mbar_wait(&sm.item_full[nth & 1], (nth >> 1) & 1, &sm.abort_flag, p.status, 133);
      if (!(ok = __all_sync(0xffffffffu, ok))) break;
      // (read again where it is needed: few registers are left beside a row of S)
      const PackedItem& it = sm.item[nth & 1];
      const int num_tiles = it.num_tiles, open_tiles = it.open_tiles;
      if (num_tiles < 0) break;
      // (rows behind the item's end are nobody's)
      auto row_valid = [&]() -> bool { return token < min(it.tokens, p.tile_tokens); };
      auto out_at = [&]() -> int64_t {
        return static_cast<int64_t>(it.q_row + token) * p.o_stride_t + (it.head + tid - token * p.pack) * p.o_stride_h;
      };
      auto store_lse = [&](float lse) {
        p.lse[static_cast<int64_t>(it.head + tid - token * p.pack) * p.total_q + it.q_row + token] = lse;
      };
      auto release_item = [&]() {
        __syncwarp();
        if (lane == 0) mbar_arrive(&sm.item_free[nth & 1]);
      };
      if (num_tiles == 0) {
        // no keys: zeros, and a log-sum-exp of -inf
        if (row_valid()) {
          uint4* o = reinterpret_cast<uint4*>(static_cast<uint16_t*>(p.o) + out_at());
          for (int i = 0; i < 16; ++i) o[i] = make_uint4(0u, 0u, 0u, 0u);
          if (p.lse != nullptr) store_lse(-INFINITY);
        }
        release_item();
        continue;
      }
      // keys this row sees
      auto keys_of_row = [&]() -> int { return it.keys_of(token, p.causal); };
      // (a row that is nobody's holds anything: a finite reference keeps it from asking for the exact path in every tile)
      RowState st{row_valid() ? -INFINITY : 0.f, 0.f};
      for (int t = 0; t < num_tiles; ++t) {
        if (t >= open_tiles) {
          // Some row of the item does not see all of these keys: V is looked at while S_t is still being worked out.
          const int g = load0 + 2 * t + 1;
          ok = mbar_wait(&sm.kv_full[g % kSlots], (g / kSlots) & 1, &sm.abort_flag, p.status, 134);
          if (!(ok = __all_sync(0xffffffffu, ok))) break;
          const int key = tid & 63;
          if (has_non_finite<Type>(sm.kv[g % kSlots][tid >> 6], key)) {
            clean_half_row<Type>(sm.kv[g % kSlots][tid >> 6], key);
            if (t * kTileN + key < it.k_len) sm.special[nth & 1] = nth;
            fence_proxy_async_smem();
          }
        }
        const int gk = load0 + 2 * t;
        ok = mbar_wait(&sm.done[gk % kSlots], (gk / kSlots) & 1, &sm.abort_flag, p.status, 130);
        if (!(ok = __all_sync(0xffffffffu, ok))) break;
        tc_fence_after();
        const int buf = (tile0 + t) & 1;
        const uint32_t tS = tmem + kColS + buf * kTileN + lane_base;
        uint32_t r0[32], r1[32], pk[32];
        tmem_ld32(tS, r0);
        tmem_ld32(tS + 32, r1);
        tmem_wait_ld();
        if (t >= open_tiles) {
          // (the rows of a warp are neighbours: the mask's edge usually runs through one half of the columns)
          const int valid = keys_of_row() - t * kTileN;
          const int least = __reduce_min_sync(0xffffffffu, valid);
          if (least < 32) mask_half(r0, valid);
          if (least < 64) mask_half(r1, valid - 32);
        }
        float2 sums = make_float2(0.f, 0.f);
        bool exact = st.m == -INFINITY;   // nothing accumulated yet: no reference maximum to try
        if (!__any_sync(0xffffffffu, exact)) {
          sums = softmax_group_fast<Type>(r0, r1, scale_log2, st.m, pk);
          exact = sums.x + sums.y > Type::kMostSum;   // logits outgrew the running maximum (a NaN makes the row NaN either way)
        }
        if (__any_sync(0xffffffffu, exact)) {
          // Rows whose reference has to move take their own maximum of the tile, less the headroom; the others keep theirs and get the same P
          // again, so that a row's result does not depend on its neighbours (later tokens, with a causal mask).
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
          // (a row whose logits so far are all -inf: 2^(-inf - 0) = 0, not NaN)
          sums = softmax_group_fast<Type>(r0, r1, scale_log2, st.m == -INFINITY ? 0.f : st.m, pk);
          if (t > 0) {
            // O must be quiescent: wait until P_{t-1} V_{t-1} (which read ring load 2t-1) has drained
            const int gp = load0 + 2 * t - 1;
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
        tc_fence_before();
        mbar_arrive(&sm.p_full[buf]);
      }
      // ---- epilogue: O / l -> 16 bits -> shared memory (the dead Q tile) -> global, each warp its own rows --------
      if (ok) {
        const int gl = load0 + 2 * num_tiles - 1;   // the last P V read this load's slot
        ok = mbar_wait(&sm.done[gl % kSlots], (gl / kSlots) & 1, &sm.abort_flag, p.status, 131);
      }
      if (!(ok = __all_sync(0xffffffffu, ok))) break;
      tc_fence_after();
      // a row of no keys has accumulated P = 0: zeros
      const float inv_l = st.l > 0.f ? (1.f / st.l) : (st.l == 0.f ? 0.f : st.l);
      stage_output_half<Type>(tO + lane_base, true, inv_l, reinterpret_cast<__nv_bfloat16*>(sm.q[0]), tid);
      stage_output_half<Type>(tO + lane_base + 64, true, inv_l, reinterpret_cast<__nv_bfloat16*>(sm.q[1]), tid);
      tc_fence_before();   // the next item's first P V overwrites O: order these reads before its hand-over
      // (all threads wrote their notes before the hand-over of the P whose P V has just been waited for)
      if (*reinterpret_cast<volatile int*>(&sm.special[nth & 1]) == nth && row_valid()) {
        add_special<Type>(p, sm.q, tid, it.k_row, open_tiles * kTileN, keys_of_row(), it.head / p.group);
      }
      __syncwarp();
      // the Q buffer is handed back as soon as the rows are in registers
      uint4 x[16];
      read_staged_rows(sm.q, warp * 32, lane, x);
      fence_proxy_async_smem();   // (the next Q comes through the async proxy)
      __syncwarp();
      if (lane == 0) mbar_arrive(&sm.q_free);
      const bool stored = row_valid();
      store_rows(p.o, stored ? out_at() : -1, lane, x);
      if (p.lse != nullptr && stored) store_lse((st.m + log2f(st.l)) * 0.69314718055994531f);
      release_item();
      load0 += 2 * num_tiles;
      tile0 += num_tiles;
    }
  }

  // ---- teardown ------------------------------------------------------------------------
  tc_fence_before();
  __syncthreads();
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
  return launch_overlapped(kernel, static_cast<long long>(p.tiles) * (p.heads_q / p.pack), p.max_ctas, kThreads, smem, stream, tq, tk, tv, p);
}

}  // namespace

int packed_heads_per_tile(int group) {
  int pack = 1;
  for (int d = 2; d <= group && d <= kTileM; ++d)
    if (group % d == 0 && kTileM / d * d >= 124) pack = d;
  return pack;
}

cudaError_t launch_attn_packed(const CUtensorMap& tq, const CUtensorMap& tk, const CUtensorMap& tv, const PackedParams& p,
                               bool fp16, cudaStream_t stream) {
  return fp16 ? launch<Fp16Type>(tq, tk, tv, p, stream) : launch<Bf16Type>(tq, tk, tv, p, stream);
}

}  // namespace sparsed
