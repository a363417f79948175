// What the kernels of attention over packed sequences share (attention_packed.cu, attention_packed_pair.cu): which rows a tile
// number stands for, masks, and V's infinities and NaN in tiles that not every row sees.
#pragma once

#include "sequences.cuh"
#include "softmax_pipeline.cuh"

namespace sparsed {

// Some consecutive tokens of one sequence, and the keys that they see.
struct PackedTokens {
  int q_row, tokens;   // first row of q and o, and how many
  int first_keys;      // causal: keys that the first token sees (may be negative), one more for each later one
  int k_row, k_len;    // the sequence's keys
  // keys that token `i` sees
  __device__ __forceinline__ int keys_of(int i, int causal) const { return causal ? min(max(first_keys + i, 0), k_len) : k_len; }
};

// The tokens of tile number `tile`, with `per_tile` tokens to a tile: sequence b has the numbers from cu_q[b] / per_tile + b on.
// Returns false for a number beyond its sequence's last tile. By a whole warp.
__device__ __forceinline__ bool packed_tokens(const PackedParams& p, int tile, int per_tile, PackedTokens& it) {
  const int seq = last_not_above(p.num_seqs, tile, [&](int b) { return __ldcg(p.cu_q + b) / per_tile + b; });
  const int2 q_rows = sequence_rows(p.cu_q, seq, p.total_q, p.status, 4);
  const int2 k_rows = sequence_rows(p.cu_k, seq, p.total_k, p.status, 5);
  const int q_len = q_rows.y - q_rows.x;
  const int q0 = (tile - (q_rows.x / per_tile + seq)) * per_tile;   // the tile's first token in its sequence
  if (q0 < 0 || q0 >= q_len) return false;
  it.q_row = q_rows.x + q0;
  it.tokens = min(per_tile, q_len - q0);
  it.k_row = k_rows.x;
  it.k_len = k_rows.y - k_rows.x;
  it.first_keys = p.causal ? q0 + 1 + it.k_len - q_len : it.k_len;
  return true;
}

// Grid number -> tile number and packed head. Heads are taken heads_per_pass at a time (their K and V stay in L2), tiles from the
// last one down: with a causal mask a sequence's last tiles are its longest.
__device__ __forceinline__ int2 packed_tile_and_head(const PackedParams& p, int number) {
  const int per_pass = p.tiles * p.heads_per_pass, pass = number / per_pass, in_pass = number - pass * per_pass;
  const int heads_here = min(p.heads_per_pass, p.heads_q / p.pack - pass * p.heads_per_pass);
  return make_int2(p.tiles - 1 - in_pass / heads_here, pass * p.heads_per_pass + in_pass % heads_here);
}

// Whether this thread's row of a 64-column half of a V tile (128 bytes a row) holds an infinity or NaN. (Volatile, as the writes
// of clean_half_row: in the CTA-pair kernel two threads look at a row, and either may clean it.)
template <class Type>
__device__ __forceinline__ bool has_non_finite(const uint16_t* half_tile, int row) {
  const uint32_t chunks = smem_u32(half_tile + row * 64);
  uint32_t found = 0;
#pragma unroll
  for (int c = 0; c < 8; ++c) {
    uint4 x;   // (rotated: rows are 128 bytes apart; the swizzle does not matter here)
    asm volatile("ld.volatile.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w) : "r"(chunks + ((c + row) & 7) * 16) : "memory");
    found |= non_finite_pair<Type>(x.x) | non_finite_pair<Type>(x.y) | non_finite_pair<Type>(x.z) | non_finite_pair<Type>(x.w);
  }
  return found != 0u;
}

// Makes it zero there.
template <class Type>
__device__ __forceinline__ void clean_half_row(uint16_t* half_tile, int row) {
  volatile uint32_t* words = reinterpret_cast<volatile uint32_t*>(half_tile + row * 64);
  for (int i = 0; i < 32; ++i) {
    const uint32_t x = words[i], bad = non_finite_pair<Type>(x);
    if (bad != 0u) words[i] = x & ((bad & 0x8000u ? 0xffff0000u : ~0u) & (bad & 0x80000000u ? 0x0000ffffu : ~0u));
  }
}

// -inf in the columns at and beyond `valid` of 32
__device__ __forceinline__ void mask_half(uint32_t (&r)[32], int valid) {
#pragma unroll
  for (int j = 0; j < 32; ++j)
    if (j >= valid) r[j] = 0xff800000u;
}

// What was taken out of V in the masked tiles, for a row whose output (16 bits, in shared memory as stage_output_half leaves it)
// begins in `tile`: a probability times an infinity or NaN is that infinity or NaN. keys [from, to) are those the row sees there.
template <class Type>
__device__ __forceinline__ void add_special(const PackedParams& p, uint16_t (&tile)[2][128 * 64], int row, int k_row, int from, int to,
                                            int kv_head) {
  for (int d = 0; d < 128; d += 2) {
    uint32_t* at = reinterpret_cast<uint32_t*>(reinterpret_cast<uint8_t*>(tile[d >> 6]) + row * 128 +
                                               ((((d & 63) >> 3) ^ (row & 7)) << 4) + (d & 7) * 2);
    float2 sum = Type::unpack(*at);
    bool any = false;
    for (int j = from; j < to; ++j) {
      const uint32_t x = __ldcg(reinterpret_cast<const uint32_t*>(static_cast<const uint16_t*>(p.v) + (k_row + j) * p.v_stride_t +
                                                                  kv_head * p.v_stride_h + d));
      const uint32_t bad = non_finite_pair<Type>(x);
      const float2 f = Type::unpack(x);
      if (bad & 0x8000u) sum.x += f.x;
      if (bad & 0x80000000u) sum.y += f.y;
      any = any || bad != 0u;
    }
    if (any) *at = Type::pack(sum.x, sum.y);
  }
}

// A warp's 32 rows of the staged output into registers: sixteen threads to a row's 256 bytes, x[i] of row 2 i + lane / 16 ...
__device__ __forceinline__ void read_staged_rows(const uint16_t (&tile)[2][128 * 64], int row0, int lane, uint4 (&x)[16]) {
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int r = row0 + 2 * i + (lane >> 4);
    x[i] = *reinterpret_cast<const uint4*>(reinterpret_cast<const uint8_t*>(tile[(lane >> 3) & 1]) + r * 128 +
                                           (((lane & 7) ^ (r & 7)) << 4));
  }
}
// ... and to global memory; `out`: element offset of this thread's own row, -1 for a row that is nobody's.
__device__ __forceinline__ void store_rows(void* o, int64_t out, int lane, const uint4 (&x)[16]) {
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int64_t to = __shfl_sync(0xffffffffu, out, 2 * i + (lane >> 4));
    if (to >= 0) *reinterpret_cast<uint4*>(static_cast<uint16_t*>(o) + to + (lane & 15) * 8) = x[i];
  }
}

}  // namespace sparsed
