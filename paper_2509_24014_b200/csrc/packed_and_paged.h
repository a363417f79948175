// Host-side interfaces of the calls on packed sequences and on a paged key-value cache.
#pragma once

#include "internal.h"

namespace sparsed {

struct PackedParams {
  const int32_t* cu_q;     // [num_seqs + 1]
  const int32_t* cu_k;
  void* o;                 // [total_q, heads_q, 128]
  int64_t o_stride_t, o_stride_h;
  const void* v;           // (only read again where it holds infinities or NaN)
  int64_t v_stride_t, v_stride_h;
  float* lse;              // fp32 [heads_q, total_q] or null
  int num_seqs, total_q, total_k, heads_q;
  int group;               // heads_q / heads_kv
  int causal;
  int pack;                // query heads of a group that share a tile (packed_heads_per_tile)
  int tile_tokens;         // 128 / pack
  int tiles;               // total_q / tile_tokens + num_seqs: numbers of query tiles, some of them empty
  int heads_per_pass;      // tiles' worth of heads that are taken before the next ones
  int max_ctas;            // CTAs that fit on the device at once (0: not known)
  float scale_log2;
  unsigned long long* slow_path_events;
  DeviceStatus* status;
};

// Query heads of a group that share a tile of 128 rows: the most that divide the group and leave at most 4 rows unused.
int packed_heads_per_tile(int group);
// (Q's tensor map: [heads_kv, total, group, 128], boxes of 64 x pack x tile_tokens; K's and V's as in attention.cu, boxes of
// 64 x 64 rows)
cudaError_t launch_attn_packed(const CUtensorMap& tq, const CUtensorMap& tk, const CUtensorMap& tv, const PackedParams& p,
                               bool fp16, cudaStream_t stream);

// The same with the MMAs spanning CTA pairs (attention_packed_pair.cu): p.tiles counts tiles of 4 * p.tile_tokens tokens, K's
// boxes are 64 x 32 rows.
cudaError_t launch_attn_packed_pair(const CUtensorMap& tq, const CUtensorMap& tk, const CUtensorMap& tv, const PackedParams& p,
                                    bool fp16, cudaStream_t stream);

// A paged cache as the kernels see it (16-bit elements).
struct CacheView {
  uint16_t *k, *v;
  const int32_t* table;
  int32_t* lens;
  int64_t table_stride;
  int64_t k_page, k_place, k_head, v_page, v_place, v_head;   // strides in elements
  int num_pages, page_shift, heads_kv, batch, max_pages;
};

struct CacheWriteParams {
  CacheView cache;
  const uint16_t *k, *v;   // [total, heads_kv, 128]
  int64_t k_token, k_head, v_token, v_head;
  const int32_t* cu;       // [batch + 1]
  int total;
  int tokens_at_once, tokens_per_warp;   // (launch_cache_write)
  DeviceStatus* status;
};
cudaError_t launch_cache_write(CacheWriteParams p, cudaStream_t stream);

// One new token per sequence (attention_paged.cu). Workspace behind the status block, in this order: PagedLayout.
struct PagedParams {
  CacheView cache;
  const uint16_t* q;
  uint16_t* o;
  int64_t q_seq, q_head, o_seq, o_head;
  float* lse;              // [batch, heads_q] or null
  const float* mass_in;    // [batch, heads_kv, mass_capacity] or null
  float* mass_out;         // ... or null
  int64_t mass_capacity;
  int group;               // query heads per key-value head
  float scale_log2;
  int ctas;                // of the main kernel
  int fills;               // whether these fill the device
  // scratch
  int32_t* prefix;         // [batch + 1] key tiles of the sequences before, for one head
  float* lse2;             // [batch, heads_q] base-2 LSE of sequences that one CTA has done by itself
  float2* part_ml;         // [2 * ctas, heads per chunk] (reference, sum) of a part
  float* part_o;           // [2 * ctas, heads per chunk, 128]
  float* logits;           // [batch, heads_q, max_pages * page_size] scaled base-2 logits, with mass_out only
  DeviceStatus* status;
};
struct PagedLayout {
  int64_t prefix, lse2, part_ml, part_o, logits, bytes;   // offsets from the workspace's start
};
PagedLayout paged_layout(int batch, int heads_kv, int group, int max_pages, int page_size, bool with_mass);
int paged_max_ctas(int batch, int heads_kv, int group, int max_pages, int page_size);   // the layout's bound on `ctas`
// (tensor maps of K and V: [pages, heads, 2, places, 64] with the two halves of head_dim apart, boxes of 64 x 16 places x 2)
cudaError_t launch_attn_paged(const CUtensorMap& tk, const CUtensorMap& tv, PagedParams p, int sms, bool fp16,
                              cudaStream_t stream);

struct EvictParams {
  CacheView from, to;
  const float* mass;       // [batch, heads_kv, mass_capacity]
  float* mass_out;         // [batch, heads_kv, mass_out_capacity]
  int64_t mass_capacity, mass_out_capacity;
  int32_t* kept;           // [batch, heads_kv, keep]
  int keep, recent;
  DeviceStatus* status;
};
cudaError_t launch_cache_evict(const EvictParams& p, cudaStream_t stream);

}  // namespace sparsed
