// C ABI of the SparseD attention library: argument validation, tensor-map construction,
// workspace layout and kernel dispatch. Declarations and contracts are in sparsed.h.
#include <atomic>
#include <cmath>
#include <cstdlib>
#include <cstring>
#include <mutex>

#include "../../include/sparsed.h"
#include "dense_choice.h"
#include "internal.h"
#include "packed_and_paged.h"

namespace {

using namespace sparsed;

thread_local int32_t g_last_cuda_error = 0;

sparsed_status cuda_fail(cudaError_t e) {
  g_last_cuda_error = static_cast<int32_t>(e);
  return SPARSED_ERR_CUDA;
}

// ---- driver entry point for tensor-map encoding (no link-time dependency on libcuda) ----
typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiledFn encode_tiled_fn() {
  static EncodeTiledFn fn = nullptr;
  static std::once_flag once;
  std::call_once(once, [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) == cudaSuccess &&
        q == cudaDriverEntryPointSuccess) {
      fn = reinterpret_cast<EncodeTiledFn>(p);
    }
  });
  return fn;
}

// Host-side cache of encoded tensor maps. A map depends only on (base pointer, extents, strides,
// box), not on the tensor's contents, so a denoising loop that calls with the same buffers every
// step encodes each map once. Per thread (no locking), direct-mapped, 32 entries.
struct TensorMapKey {
  const void* base;
  int64_t strides[3];
  int32_t batch, heads, seq_len, box_rows;
  bool operator==(const TensorMapKey& o) const {
    return base == o.base && strides[0] == o.strides[0] && strides[1] == o.strides[1] && strides[2] == o.strides[2] &&
           batch == o.batch && heads == o.heads && seq_len == o.seq_len && box_rows == o.box_rows;
  }
};
struct TensorMapSlot {
  TensorMapKey key;
  CUtensorMap map;
  bool valid;
};
constexpr int kTensorMapSlots = 32;
thread_local TensorMapSlot g_tensor_maps[kTensorMapSlots] = {};

uint32_t tensor_map_slot(const TensorMapKey& k) {
  uint64_t h = reinterpret_cast<uintptr_t>(k.base) >> 4;
  h = h * 0x9E3779B97F4A7C15ull + static_cast<uint64_t>(k.strides[1]);
  h = h * 0x9E3779B97F4A7C15ull + static_cast<uint64_t>(k.strides[2]);
  h = h * 0x9E3779B97F4A7C15ull + (static_cast<uint64_t>(k.seq_len) << 8 | static_cast<uint64_t>(k.box_rows));
  h = h * 0x9E3779B97F4A7C15ull + (static_cast<uint64_t>(k.heads) << 16 | static_cast<uint64_t>(k.batch));
  return static_cast<uint32_t>(h >> 40) % kTensorMapSlots;
}

// Any map of 16-bit elements with 128-byte swizzle.
sparsed_status encode_swizzled_map(CUtensorMap* out, const void* base, int rank, const cuuint64_t* dims,
                                   const cuuint64_t* stride_bytes, const cuuint32_t* box) {
  EncodeTiledFn enc = encode_tiled_fn();
  if (enc == nullptr) return cuda_fail(cudaErrorNotSupported);
  const cuuint32_t elem[5] = {1, 1, 1, 1, 1};
  CUresult r = enc(out, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, static_cast<cuuint32_t>(rank), const_cast<void*>(base), dims,
                   stride_bytes, box, elem, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                   CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (r != CUDA_SUCCESS) {
    g_last_cuda_error = static_cast<int32_t>(r);
    return SPARSED_ERR_CUDA;
  }
  return SPARSED_OK;
}

// bf16 [B,H,L,128] tensor with element strides (batch, head, token); box = 64 x rows, 128B swizzle.
sparsed_status make_tensor_map(CUtensorMap* out, const void* base, int batch, int heads, int seq_len,
                               const int64_t strides[3], int box_rows) {
  TensorMapKey key{base, {strides[0], strides[1], strides[2]}, batch, heads, seq_len, box_rows};
  TensorMapSlot& slot = g_tensor_maps[tensor_map_slot(key)];
  if (slot.valid && slot.key == key) {
    *out = slot.map;
    return SPARSED_OK;
  }
  cuuint64_t dims[4] = {128, static_cast<cuuint64_t>(seq_len), static_cast<cuuint64_t>(heads),
                        static_cast<cuuint64_t>(batch)};
  cuuint64_t gstrides[3] = {static_cast<cuuint64_t>(strides[2]) * 2, static_cast<cuuint64_t>(strides[1]) * 2,
                            static_cast<cuuint64_t>(strides[0]) * 2};
  cuuint32_t box[4] = {64, static_cast<cuuint32_t>(box_rows), 1, 1};
  const sparsed_status st = encode_swizzled_map(out, base, 4, dims, gstrides, box);
  if (st != SPARSED_OK) return st;
  slot.key = key;
  slot.map = *out;
  slot.valid = true;
  return SPARSED_OK;
}

// The maps of the packed and paged calls are encoded anew for every call.
// Packed keys or values, [total, heads, 128] with element strides (token, head), under a batch of one as above; box = 64 x
// box_rows tokens.
sparsed_status make_packed_key_map(CUtensorMap* out, const void* base, int total, int heads, const int64_t strides[2], int box_rows) {
  const cuuint64_t dims[4] = {128, static_cast<cuuint64_t>(total), static_cast<cuuint64_t>(heads), 1};
  const cuuint64_t token = static_cast<cuuint64_t>(strides[0]) * 2, head = static_cast<cuuint64_t>(strides[1]) * 2;
  const cuuint64_t stride_bytes[3] = {token, head, token};
  const cuuint32_t box[4] = {64, static_cast<cuuint32_t>(box_rows), 1, 1};
  return encode_swizzled_map(out, base, 4, dims, stride_bytes, box);
}

// One pool of a paged cache, [pages, places, heads, 128] with element strides (page, place, head), as [pages, heads, 2 halves,
// places, 64]; box = 64 x 16 places x both halves.
sparsed_status make_pool_map(CUtensorMap* out, const void* base, int pages, int places, int heads, int64_t page_stride,
                             int64_t place_stride, int64_t head_stride) {
  const cuuint64_t dims[5] = {64, static_cast<cuuint64_t>(places), 2, static_cast<cuuint64_t>(heads), static_cast<cuuint64_t>(pages)};
  const cuuint64_t strides[4] = {static_cast<cuuint64_t>(place_stride) * 2, 128, static_cast<cuuint64_t>(head_stride) * 2,
                                 static_cast<cuuint64_t>(page_stride) * 2};
  const cuuint32_t box[5] = {64, 16, 2, 1, 1};
  return encode_swizzled_map(out, base, 5, dims, strides, box);
}

// Packed queries, [total, heads, 128] with element strides (token, head), as [key-value heads, total, heads of a group, 128];
// box = 64 x `pack` heads x `tokens`.
sparsed_status make_packed_query_map(CUtensorMap* out, const void* base, int total, int heads_kv, int group, int64_t token_stride,
                                     int64_t head_stride, int pack, int tokens) {
  const cuuint64_t dims[4] = {128, static_cast<cuuint64_t>(group), static_cast<cuuint64_t>(total), static_cast<cuuint64_t>(heads_kv)};
  const cuuint64_t strides[3] = {static_cast<cuuint64_t>(head_stride) * 2, static_cast<cuuint64_t>(token_stride) * 2,
                                 static_cast<cuuint64_t>(head_stride) * 2 * group};
  const cuuint32_t box[4] = {64, static_cast<cuuint32_t>(pack), static_cast<cuuint32_t>(tokens), 1};
  return encode_swizzled_map(out, base, 4, dims, strides, box);
}

struct Resolved {
  int64_t q[3], k[3], v[3], o[3];
  float scale_log2;
};

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

// The workspace holds the status word (atomics) and fp32 arrays the kernels read with 16-byte loads.
sparsed_status check_ws(const void* ws, size_t ws_bytes, size_t need) {
  if (ws == nullptr || ws_bytes < need) return SPARSED_ERR_WORKSPACE;
  return aligned16(ws) ? SPARSED_OK : SPARSED_ERR_ALIGNMENT;
}

void default_strides(const int64_t in[3], int heads, int seq_len, int64_t out[3]) {
  if (in[0] == 0 && in[1] == 0 && in[2] == 0) {
    out[2] = 128;
    out[1] = static_cast<int64_t>(seq_len) * 128;
    out[0] = out[1] * heads;
  } else {
    out[0] = in[0];
    out[1] = in[1];
    out[2] = in[2];
  }
}

sparsed_status check_arch() {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return cuda_fail(e);
  static std::atomic<int> cached_major[64];  // 0 = not looked up yet
  int major = (dev >= 0 && dev < 64) ? cached_major[dev].load(std::memory_order_relaxed) : 0;
  if (major == 0) {
    e = cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev);
    if (e != cudaSuccess) return cuda_fail(e);
    if (dev >= 0 && dev < 64) cached_major[dev].store(major, std::memory_order_relaxed);
  }
  return major == 10 ? SPARSED_OK : SPARSED_ERR_ARCH;
}

// CTAs of the single-CTA attention kernel, or of the scoring kernel, that are resident on the current device at once
// (two per SM), cached per device; 0 if the SM count cannot be read (the attention kernel then gets one CTA per query
// tile).
int attn_max_ctas() {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return 0;
  static std::atomic<int> cached[64];
  int n = (dev >= 0 && dev < 64) ? cached[dev].load(std::memory_order_relaxed) : 0;
  if (n == 0) {
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
    if (dev >= 0 && dev < 64) cached[dev].store(n, std::memory_order_relaxed);
  }
  return 2 * n;
}

sparsed_status check_shape(const sparsed_shape* s, bool need_v_o, Resolved* r) {
  if (s == nullptr) return SPARSED_ERR_INVALID_ARG;
  if (s->batch < 1 || s->heads_q < 1 || s->heads_kv < 1 || s->seq_len < 1) return SPARSED_ERR_INVALID_ARG;
  if (s->heads_q % s->heads_kv != 0) return SPARSED_ERR_INVALID_ARG;
  if (s->head_dim != 128) return SPARSED_ERR_UNSUPPORTED;
  if (!(s->softmax_scale >= 0.f) || !std::isfinite(s->softmax_scale)) return SPARSED_ERR_INVALID_ARG;
  default_strides(s->q_strides, s->heads_q, s->seq_len, r->q);
  default_strides(s->k_strides, s->heads_kv, s->seq_len, r->k);
  default_strides(s->v_strides, s->heads_kv, s->seq_len, r->v);
  default_strides(s->o_strides, s->heads_q, s->seq_len, r->o);
  const int64_t* sets[4] = {r->q, r->k, r->v, r->o};
  for (int t = 0; t < (need_v_o ? 4 : 2); ++t) {
    for (int i = 0; i < 3; ++i) {
      if (sets[t][i] <= 0) return SPARSED_ERR_INVALID_ARG;
      if (sets[t][i] % 8 != 0) return SPARSED_ERR_ALIGNMENT;
    }
    if (sets[t][2] < 128) return SPARSED_ERR_INVALID_ARG;
  }
  const float scale = s->softmax_scale == 0.f ? 1.0f / std::sqrt(static_cast<float>(s->head_dim)) : s->softmax_scale;
  r->scale_log2 = scale * 1.44269504088896341f;
  return SPARSED_OK;
}

sparsed_status kept_counts(const sparsed_select_params* sp, int nb, int* pb, int* k_pre, int* k_gen) {
  if (sp == nullptr) return SPARSED_ERR_INVALID_ARG;
  if (sp->block_size != 32 && sp->block_size != 64 && sp->block_size != 128) return SPARSED_ERR_UNSUPPORTED;
  if (!(sp->keep_ratio > 0.0) || !(sp->keep_ratio <= 1.0)) return SPARSED_ERR_INVALID_ARG;
  if (sp->rounding != 0 && sp->rounding != 1) return SPARSED_ERR_INVALID_ARG;
  if (sp->prefill_len < 0) return SPARSED_ERR_INVALID_ARG;
  if (sp->prefill_len % sp->block_size != 0) return SPARSED_ERR_ALIGNMENT;
  const int p_blocks = sp->prefill_len / sp->block_size;
  if (p_blocks > nb) return SPARSED_ERR_INVALID_ARG;
  auto kept = [&](int n) -> int {
    if (n <= 0) return 0;
    const double x = sp->keep_ratio * n;
    long long kk = sp->rounding == 0 ? static_cast<long long>(std::ceil(x - 1e-6))
                                     : static_cast<long long>(std::floor(x + 1e-6));
    if (kk < 1) kk = 1;
    if (kk > n) kk = n;
    return static_cast<int>(kk);
  };
  *pb = p_blocks;
  *k_pre = kept(p_blocks);
  *k_gen = kept(nb - p_blocks);
  return SPARSED_OK;
}

size_t round_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

// Whether the switch step can select from the row statistics of its own full-attention pass.
bool step_uses_stats(const sparsed_shape* shape, const sparsed_select_params* params) {
  return shape->seq_len / params->block_size <= pool_select_max_blocks();
}

// Checks the caller's pattern buffers against the number of rows and kept blocks per row and
// fills in the host-side fields of `out`.
sparsed_status prepare_pattern(sparsed_pattern* out, int batch, int heads_q, int nb, int block_size, int k_total) {
  if (out == nullptr || out->row_ptr == nullptr || out->col_idx == nullptr) return SPARSED_ERR_PATTERN;
  if (!aligned4(out->row_ptr) || !aligned4(out->col_idx)) return SPARSED_ERR_ALIGNMENT;
  if (nb > 16384) return SPARSED_ERR_UNSUPPORTED;
  const int64_t rows = static_cast<int64_t>(batch) * heads_q * nb;
  const int64_t nnz = rows * k_total;
  if (rows >= INT32_MAX || nnz >= INT32_MAX) return SPARSED_ERR_UNSUPPORTED;
  if (out->col_capacity < nnz) return SPARSED_ERR_PATTERN;
  out->nnz = nnz;
  out->block_size = block_size;
  out->num_blocks = nb;
  out->batch = batch;
  out->heads_q = heads_q;
  return SPARSED_OK;
}

sparsed_status run_topk(const float* scores, int batch, int heads_q, int nb, int block_size, int pb, int k_pre,
                        int k_gen, sparsed_pattern* out, cudaStream_t stream) {
  sparsed_status st = prepare_pattern(out, batch, heads_q, nb, block_size, k_pre + k_gen);
  if (st != SPARSED_OK) return st;
  TopkParams tp;
  tp.scores = scores;
  tp.row_ptr = out->row_ptr;
  tp.col_idx = out->col_idx;
  tp.rows = batch * heads_q * nb;
  tp.nb = nb;
  tp.pb = pb;
  tp.k_pre = k_pre;
  tp.k_gen = k_gen;
  cudaError_t e = launch_topk_csr(tp, stream);
  if (e != cudaSuccess) return cuda_fail(e);
  return SPARSED_OK;
}

}  // namespace

extern "C" {

const char* sparsed_status_string(sparsed_status status) {
  switch (status) {
    case SPARSED_OK: return "ok";
    case SPARSED_ERR_INVALID_ARG: return "invalid argument";
    case SPARSED_ERR_UNSUPPORTED: return "unsupported configuration";
    case SPARSED_ERR_ALIGNMENT: return "alignment or divisibility requirement not met";
    case SPARSED_ERR_WORKSPACE: return "workspace missing or too small";
    case SPARSED_ERR_PATTERN: return "pattern invalid or too small";
    case SPARSED_ERR_ARCH: return "device is not compute capability 10.x";
    case SPARSED_ERR_CUDA: return "CUDA error";
    case SPARSED_ERR_DEVICE_TIMEOUT: return "device-side wait ran out";
  }
  return "unknown status";
}

int32_t sparsed_last_cuda_error(void) { return g_last_cuda_error; }

int32_t sparsed_switch_step(int32_t total_steps, double skip) {
  if (total_steps < 1 || !(skip >= 0.0) || !(skip <= 1.0)) return -1;
  long long s = static_cast<long long>(std::floor(static_cast<double>(total_steps) * skip + 1e-9));
  if (s < 1) s = 1;
  if (s > total_steps) s = total_steps;
  return static_cast<int32_t>(s);
}

int32_t sparsed_schedule_mode(int32_t step_1based, int32_t total_steps, double skip) {
  const int32_t s = sparsed_switch_step(total_steps, skip);
  if (s < 0 || step_1based < 1 || step_1based > total_steps) return -1;
  if (step_1based < s) return SPARSED_MODE_FULL;
  if (step_1based == s) return SPARSED_MODE_FULL_AND_SELECT;
  return SPARSED_MODE_SPARSE;
}

sparsed_status sparsed_kept_per_row(const sparsed_select_params* params, int32_t seq_len, int32_t* k_pre,
                                    int32_t* k_gen) {
  if (params == nullptr || k_pre == nullptr || k_gen == nullptr || seq_len < 1) return SPARSED_ERR_INVALID_ARG;
  if (params->block_size != 32 && params->block_size != 64 && params->block_size != 128) return SPARSED_ERR_UNSUPPORTED;
  if (seq_len % params->block_size != 0) return SPARSED_ERR_ALIGNMENT;
  int pb = 0, a = 0, b = 0;
  sparsed_status st = kept_counts(params, seq_len / params->block_size, &pb, &a, &b);
  if (st != SPARSED_OK) return st;
  *k_pre = a;
  *k_gen = b;
  return SPARSED_OK;
}

sparsed_status sparsed_workspace_bytes(int32_t op, const sparsed_shape* shape, const sparsed_select_params* params,
                                       size_t* out_bytes) {
  if (out_bytes == nullptr) return SPARSED_ERR_INVALID_ARG;
  switch (op) {
    case SPARSED_OP_ATTN_FULL:
    case SPARSED_OP_ATTN_SPARSE:
    case SPARSED_OP_SELECT_FROM_SCORES:
    case SPARSED_OP_PATTERN_VALIDATE:
    case SPARSED_OP_ATTN_PACKED:
    case SPARSED_OP_CACHE_WRITE:
      *out_bytes = SPARSED_STATUS_BYTES;
      return SPARSED_OK;
    case SPARSED_OP_SELECT_PATTERN: {
      if (shape == nullptr || params == nullptr) return SPARSED_ERR_INVALID_ARG;
      if (params->block_size != 32 && params->block_size != 64 && params->block_size != 128) return SPARSED_ERR_UNSUPPORTED;
      if (shape->batch < 1 || shape->heads_q < 1 || shape->seq_len < 1) return SPARSED_ERR_INVALID_ARG;
      if (shape->seq_len % params->block_size != 0) return SPARSED_ERR_ALIGNMENT;
      const size_t nb = static_cast<size_t>(shape->seq_len / params->block_size);
      const size_t bh = static_cast<size_t>(shape->batch) * shape->heads_q;
      *out_bytes = SPARSED_STATUS_BYTES + round_up(bh * nb * nb * 4, 256) +
                   round_up(bh * static_cast<size_t>(shape->seq_len) * 4, 256);
      return SPARSED_OK;
    }
    case SPARSED_OP_SELECT_POOLED_QK: {
      if (shape == nullptr || params == nullptr) return SPARSED_ERR_INVALID_ARG;
      if (params->block_size != 32 && params->block_size != 64 && params->block_size != 128) return SPARSED_ERR_UNSUPPORTED;
      if (shape->batch < 1 || shape->heads_q < 1 || shape->heads_kv < 1 || shape->seq_len < 1) return SPARSED_ERR_INVALID_ARG;
      if (shape->seq_len % params->block_size != 0) return SPARSED_ERR_ALIGNMENT;
      *out_bytes = SPARSED_STATUS_BYTES +
                   pooled_qk_means_bytes(shape->batch, shape->heads_q, shape->heads_kv, shape->seq_len / params->block_size);
      return SPARSED_OK;
    }
    case SPARSED_OP_ATTENTION_STEP: {
      if (shape == nullptr || params == nullptr) return SPARSED_ERR_INVALID_ARG;
      if (params->block_size != 32 && params->block_size != 64 && params->block_size != 128) return SPARSED_ERR_UNSUPPORTED;
      if (shape->batch < 1 || shape->heads_q < 1 || shape->seq_len < 1) return SPARSED_ERR_INVALID_ARG;
      if (shape->seq_len % params->block_size != 0) return SPARSED_ERR_ALIGNMENT;
      const size_t nb = static_cast<size_t>(shape->seq_len / params->block_size);
      const size_t bh = static_cast<size_t>(shape->batch) * shape->heads_q;
      const size_t lse_bytes = round_up(bh * static_cast<size_t>(shape->seq_len) * 4, 256);
      if (step_uses_stats(shape, params)) {
        size_t stats = 0;
        sparsed_status st = sparsed_tile_stats_bytes(shape, params->block_size, &stats);
        if (st != SPARSED_OK) return st;
        *out_bytes = SPARSED_STATUS_BYTES + lse_bytes + stats;
      } else {
        *out_bytes = SPARSED_STATUS_BYTES + round_up(bh * nb * nb * 4, 256) + lse_bytes;
      }
      return SPARSED_OK;
    }
    default:
      return SPARSED_ERR_INVALID_ARG;
  }
}

sparsed_status sparsed_workspace_init(void* ws, size_t ws_bytes, void* cuda_stream) {
  sparsed_status st = check_ws(ws, ws_bytes, SPARSED_STATUS_BYTES);
  if (st != SPARSED_OK) return st;
  cudaError_t e = cudaMemsetAsync(ws, 0, SPARSED_STATUS_BYTES, static_cast<cudaStream_t>(cuda_stream));
  return e == cudaSuccess ? SPARSED_OK : cuda_fail(e);
}

// Which dense kernel runs. The environment variable SPARSED_DENSE_KERNEL (read once) sends every pass to one of them,
// `pair`, `single` or `lone`, for A/B measurements and tests; a pass that records row statistics, which the single-CTA
// kernel cannot do, is not sent there.
static DenseKernel dense_kernel(bool with_stats, const sparsed_shape* shape, int max_ctas) {
  static const int forced = [] {
    const char* v = std::getenv("SPARSED_DENSE_KERNEL");
    if (v != nullptr && std::strcmp(v, "pair") == 0) return static_cast<int>(DenseKernel::kPair);
    if (v != nullptr && std::strcmp(v, "single") == 0) return static_cast<int>(DenseKernel::kSingle);
    if (v != nullptr && std::strcmp(v, "lone") == 0) return static_cast<int>(DenseKernel::kLone);
    return -1;
  }();
  if (forced >= 0 && !(with_stats && forced == static_cast<int>(DenseKernel::kSingle)))
    return static_cast<DenseKernel>(forced);
  return choose_dense_kernel(with_stats, static_cast<long long>(shape->batch) * shape->heads_q, shape->seq_len, max_ctas);
}

static sparsed_status attn_full_impl(const sparsed_shape* shape, const void* q, const void* k, const void* v, void* o,
                                     float* lse_or_null, float* tile_lse_or_null, int stat_keys, void* ws,
                                     size_t ws_bytes, void* cuda_stream) {
  Resolved rs;
  sparsed_status st = check_shape(shape, true, &rs);
  if (st != SPARSED_OK) return st;
  if (q == nullptr || k == nullptr || v == nullptr || o == nullptr) return SPARSED_ERR_INVALID_ARG;
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(o)) return SPARSED_ERR_ALIGNMENT;
  if (!aligned16(lse_or_null) || !aligned16(tile_lse_or_null)) return SPARSED_ERR_ALIGNMENT;
  if ((st = check_ws(ws, ws_bytes, SPARSED_STATUS_BYTES)) != SPARSED_OK) return st;
  if ((st = check_arch()) != SPARSED_OK) return st;
  const int max_ctas = attn_max_ctas();
  const DenseKernel kernel = dense_kernel(tile_lse_or_null != nullptr, shape, max_ctas);
  CUtensorMap tq, tk, tv, to;
  if ((st = make_tensor_map(&tq, q, shape->batch, shape->heads_q, shape->seq_len, rs.q, 128)) != SPARSED_OK) return st;
  if ((st = make_tensor_map(&to, o, shape->batch, shape->heads_q, shape->seq_len, rs.o, 128)) != SPARSED_OK) return st;
  const int k_box = kernel == DenseKernel::kPair ? 32 : 64;
  if ((st = make_tensor_map(&tk, k, shape->batch, shape->heads_kv, shape->seq_len, rs.k, k_box)) != SPARSED_OK) return st;
  if ((st = make_tensor_map(&tv, v, shape->batch, shape->heads_kv, shape->seq_len, rs.v, 64)) != SPARSED_OK) return st;
  AttnParams p;
  p.o = o;
  p.o_stride_b = rs.o[0];
  p.o_stride_h = rs.o[1];
  p.o_stride_t = rs.o[2];
  p.lse = lse_or_null;
  p.tile_lse = tile_lse_or_null;
  p.stat_keys = stat_keys;
  p.slow_path_events = reinterpret_cast<unsigned long long*>(static_cast<uint8_t*>(ws) + 32);
  p.seq_len = shape->seq_len;
  p.heads_q = shape->heads_q;
  p.group = shape->heads_q / shape->heads_kv;
  p.num_q_tiles = (shape->seq_len + 127) / 128;
  p.num_blocks = 0;
  p.num_items = shape->batch * shape->heads_q * p.num_q_tiles;
  p.max_ctas = max_ctas;
  p.scale_log2 = rs.scale_log2;
  p.row_ptr = nullptr;
  p.col_idx = nullptr;
  p.col_capacity = 0;
  p.status = static_cast<DeviceStatus*>(ws);
  const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  cudaError_t e = kernel == DenseKernel::kPair   ? launch_attn_dense_pair(tq, tk, tv, to, p, stream)
                  : kernel == DenseKernel::kLone ? launch_attn_dense_lone(tq, tk, tv, p, stream)
                                                 : launch_attn_dense(tq, tk, tv, to, p, stream);
  return e == cudaSuccess ? SPARSED_OK : cuda_fail(e);
}

sparsed_status sparsed_attn_full(const sparsed_shape* shape, const void* q, const void* k, const void* v, void* o,
                                 float* lse_or_null, void* ws, size_t ws_bytes, void* cuda_stream) {
  return attn_full_impl(shape, q, k, v, o, lse_or_null, nullptr, 64, ws, ws_bytes, cuda_stream);
}

sparsed_status sparsed_tile_stats_bytes(const sparsed_shape* shape, int32_t block_size, size_t* out_bytes) {
  if (shape == nullptr || out_bytes == nullptr) return SPARSED_ERR_INVALID_ARG;
  if (shape->batch < 1 || shape->heads_q < 1 || shape->seq_len < 1) return SPARSED_ERR_INVALID_ARG;
  if (block_size != 32 && block_size != 64 && block_size != 128) return SPARSED_ERR_UNSUPPORTED;
  if (shape->seq_len % block_size != 0) return SPARSED_ERR_ALIGNMENT;
  const size_t groups = static_cast<size_t>(shape->seq_len / block_size);
  const size_t q_tiles = (static_cast<size_t>(shape->seq_len) + 127) / 128;
  *out_bytes = static_cast<size_t>(shape->batch) * shape->heads_q * q_tiles * groups * 128 * 4;
  return SPARSED_OK;
}

sparsed_status sparsed_attn_full_stats(const sparsed_shape* shape, int32_t block_size, const void* q, const void* k,
                                       const void* v, void* o, float* lse, float* tile_stats, void* ws,
                                       size_t ws_bytes, void* cuda_stream) {
  if (shape == nullptr || lse == nullptr || tile_stats == nullptr) return SPARSED_ERR_INVALID_ARG;
  if (block_size != 32 && block_size != 64 && block_size != 128) return SPARSED_ERR_UNSUPPORTED;
  if (shape->seq_len >= 1 && shape->seq_len % block_size != 0) return SPARSED_ERR_ALIGNMENT;
  return attn_full_impl(shape, q, k, v, o, lse, tile_stats, block_size, ws, ws_bytes, cuda_stream);
}

sparsed_status sparsed_select_from_stats(const sparsed_shape* shape, const sparsed_select_params* params,
                                         const float* lse, const float* tile_stats, sparsed_pattern* out,
                                         float* scores_out_or_null, void* ws, size_t ws_bytes, void* cuda_stream) {
  if (shape == nullptr || params == nullptr) return SPARSED_ERR_INVALID_ARG;
  if (shape->batch < 1 || shape->heads_q < 1 || shape->seq_len < 1) return SPARSED_ERR_INVALID_ARG;
  if (params->block_size != 32 && params->block_size != 64 && params->block_size != 128) return SPARSED_ERR_UNSUPPORTED;
  if (shape->seq_len % params->block_size != 0) return SPARSED_ERR_ALIGNMENT;
  const int nb = shape->seq_len / params->block_size;
  int pb = 0, k_pre = 0, k_gen = 0;
  sparsed_status st = kept_counts(params, nb, &pb, &k_pre, &k_gen);
  if (st != SPARSED_OK) return st;
  if (lse == nullptr || tile_stats == nullptr) return SPARSED_ERR_INVALID_ARG;
  if (!aligned16(lse) || !aligned16(tile_stats) || !aligned16(scores_out_or_null)) return SPARSED_ERR_ALIGNMENT;
  if (nb > pool_select_max_blocks()) return SPARSED_ERR_UNSUPPORTED;
  if ((st = prepare_pattern(out, shape->batch, shape->heads_q, nb, params->block_size, k_pre + k_gen)) != SPARSED_OK)
    return st;
  if ((st = check_ws(ws, ws_bytes, SPARSED_STATUS_BYTES)) != SPARSED_OK) return st;
  if ((st = check_arch()) != SPARSED_OK) return st;
  PoolParams pp;
  pp.tile_lse = tile_stats;
  pp.lse = lse;
  pp.scores = scores_out_or_null;
  pp.row_ptr = out->row_ptr;
  pp.col_idx = out->col_idx;
  pp.seq_len = shape->seq_len;
  pp.block_size = params->block_size;
  pp.pb = pb;
  pp.k_pre = k_pre;
  pp.k_gen = k_gen;
  pp.bh = shape->batch * shape->heads_q;
  cudaError_t e = launch_pool_select(pp, static_cast<cudaStream_t>(cuda_stream));
  return e == cudaSuccess ? SPARSED_OK : cuda_fail(e);
}

sparsed_status sparsed_select_pattern_pooled_qk(const sparsed_shape* shape, const sparsed_select_params* params,
                                                const void* q, const void* k, sparsed_pattern* out,
                                                float* scores_out_or_null, void* ws, size_t ws_bytes,
                                                void* cuda_stream) {
  Resolved rs;
  sparsed_status st = check_shape(shape, false, &rs);
  if (st != SPARSED_OK) return st;
  if (params == nullptr) return SPARSED_ERR_INVALID_ARG;
  if (q == nullptr || k == nullptr) return SPARSED_ERR_INVALID_ARG;
  if (!aligned16(q) || !aligned16(k) || !aligned16(scores_out_or_null)) return SPARSED_ERR_ALIGNMENT;
  if (params->block_size != 32 && params->block_size != 64 && params->block_size != 128) return SPARSED_ERR_UNSUPPORTED;
  if (shape->seq_len % params->block_size != 0) return SPARSED_ERR_ALIGNMENT;
  const int nb = shape->seq_len / params->block_size;
  int pb = 0, k_pre = 0, k_gen = 0;
  if ((st = kept_counts(params, nb, &pb, &k_pre, &k_gen)) != SPARSED_OK) return st;
  if (nb > kPooledQkMaxBlocks) return SPARSED_ERR_UNSUPPORTED;
  if ((st = prepare_pattern(out, shape->batch, shape->heads_q, nb, params->block_size, k_pre + k_gen)) != SPARSED_OK)
    return st;
  size_t need = 0;
  if ((st = sparsed_workspace_bytes(SPARSED_OP_SELECT_POOLED_QK, shape, params, &need)) != SPARSED_OK) return st;
  if ((st = check_ws(ws, ws_bytes, need)) != SPARSED_OK) return st;
  if ((st = check_arch()) != SPARSED_OK) return st;
  PooledQkParams p;
  p.q = q;
  p.k = k;
  p.q_stride_b = rs.q[0];
  p.q_stride_h = rs.q[1];
  p.q_stride_t = rs.q[2];
  p.k_stride_b = rs.k[0];
  p.k_stride_h = rs.k[1];
  p.k_stride_t = rs.k[2];
  p.means = reinterpret_cast<float*>(static_cast<uint8_t*>(ws) + SPARSED_STATUS_BYTES);
  p.scores = scores_out_or_null;
  p.row_ptr = out->row_ptr;
  p.col_idx = out->col_idx;
  p.batch = shape->batch;
  p.heads_q = shape->heads_q;
  p.group = shape->heads_q / shape->heads_kv;
  p.nb = nb;
  p.block_size = params->block_size;
  p.pb = pb;
  p.k_pre = k_pre;
  p.k_gen = k_gen;
  p.scale_log2 = rs.scale_log2;
  cudaError_t e = launch_pooled_qk_select(p, static_cast<cudaStream_t>(cuda_stream));
  return e == cudaSuccess ? SPARSED_OK : cuda_fail(e);
}

sparsed_status sparsed_attn_sparse(const sparsed_shape* shape, const sparsed_pattern* pattern, const void* q,
                                   const void* k, const void* v, void* o, void* ws, size_t ws_bytes,
                                   void* cuda_stream) {
  Resolved rs;
  sparsed_status st = check_shape(shape, true, &rs);
  if (st != SPARSED_OK) return st;
  if (q == nullptr || k == nullptr || v == nullptr || o == nullptr) return SPARSED_ERR_INVALID_ARG;
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(o)) return SPARSED_ERR_ALIGNMENT;
  if (pattern == nullptr || pattern->row_ptr == nullptr || pattern->col_idx == nullptr) return SPARSED_ERR_PATTERN;
  if (!aligned4(pattern->row_ptr) || !aligned4(pattern->col_idx)) return SPARSED_ERR_ALIGNMENT;
  if (pattern->block_size != 32 && pattern->block_size != 64 && pattern->block_size != 128) return SPARSED_ERR_UNSUPPORTED;
  if (pattern->batch != shape->batch || pattern->heads_q != shape->heads_q || pattern->num_blocks < 1 ||
      static_cast<int64_t>(pattern->num_blocks) * pattern->block_size != shape->seq_len)
    return SPARSED_ERR_PATTERN;
  if ((st = check_ws(ws, ws_bytes, SPARSED_STATUS_BYTES)) != SPARSED_OK) return st;
  if ((st = check_arch()) != SPARSED_OK) return st;
  const int bs = pattern->block_size;
  if (pattern->num_blocks > attn_sparse_max_blocks(bs)) return SPARSED_ERR_UNSUPPORTED;
  CUtensorMap tq, tk, tv, to;
  if ((st = make_tensor_map(&tq, q, shape->batch, shape->heads_q, shape->seq_len, rs.q, 128)) != SPARSED_OK) return st;
  if ((st = make_tensor_map(&to, o, shape->batch, shape->heads_q, shape->seq_len, rs.o, 128)) != SPARSED_OK) return st;
  const int kv_box = bs < 64 ? bs : 64;
  if ((st = make_tensor_map(&tk, k, shape->batch, shape->heads_kv, shape->seq_len, rs.k, kv_box)) != SPARSED_OK) return st;
  if ((st = make_tensor_map(&tv, v, shape->batch, shape->heads_kv, shape->seq_len, rs.v, kv_box)) != SPARSED_OK) return st;
  AttnParams p;
  p.o = o;
  p.o_stride_b = rs.o[0];
  p.o_stride_h = rs.o[1];
  p.o_stride_t = rs.o[2];
  p.lse = nullptr;
  p.tile_lse = nullptr;
  p.stat_keys = 64;
  p.slow_path_events = reinterpret_cast<unsigned long long*>(static_cast<uint8_t*>(ws) + 32);
  p.seq_len = shape->seq_len;
  p.heads_q = shape->heads_q;
  p.group = shape->heads_q / shape->heads_kv;
  p.num_q_tiles = (shape->seq_len + 127) / 128;
  p.num_blocks = pattern->num_blocks;
  p.num_items = shape->batch * shape->heads_q * p.num_q_tiles;
  // 128-key blocks: as many CTAs as are resident at once, each running through its share of the query tiles, so
  // that only a CTA's first tile pays the start-up chain (+16 % at 4 blocks per row, +5 % at 14, +1 % at 52)
  p.max_ctas = attn_max_ctas();
  p.scale_log2 = rs.scale_log2;
  p.row_ptr = pattern->row_ptr;
  p.col_idx = pattern->col_idx;
  p.col_capacity = pattern->col_capacity;
  p.status = static_cast<DeviceStatus*>(ws);
  const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  const long long rows = static_cast<long long>(shape->batch) * shape->heads_q * pattern->num_blocks;
  const bool lone = sparse_lone_ctas_pay(p.num_items, pattern->nnz, rows, pattern->num_blocks, bs, p.max_ctas);
  cudaError_t e = lone ? launch_attn_sparse_lone(tq, tk, tv, p, bs, stream)
                       : launch_attn_sparse(tq, tk, tv, to, p, bs, stream);
  return e == cudaSuccess ? SPARSED_OK : cuda_fail(e);
}

sparsed_status sparsed_select_from_scores(const sparsed_select_params* params, const float* scores, int32_t batch,
                                          int32_t heads_q, int32_t num_blocks, sparsed_pattern* out, void* ws,
                                          size_t ws_bytes, void* cuda_stream) {
  if (scores == nullptr || batch < 1 || heads_q < 1 || num_blocks < 1) return SPARSED_ERR_INVALID_ARG;
  if (!aligned16(scores)) return SPARSED_ERR_ALIGNMENT;
  int pb = 0, k_pre = 0, k_gen = 0;
  sparsed_status st = kept_counts(params, num_blocks, &pb, &k_pre, &k_gen);
  if (st != SPARSED_OK) return st;
  if ((st = check_ws(ws, ws_bytes, SPARSED_STATUS_BYTES)) != SPARSED_OK) return st;
  if (out == nullptr || out->row_ptr == nullptr || out->col_idx == nullptr) return SPARSED_ERR_PATTERN;
  if ((st = check_arch()) != SPARSED_OK) return st;
  return run_topk(scores, batch, heads_q, num_blocks, params->block_size, pb, k_pre, k_gen, out,
                  static_cast<cudaStream_t>(cuda_stream));
}

sparsed_status sparsed_select_pattern(const sparsed_shape* shape, const sparsed_select_params* params, const void* q,
                                      const void* k, const float* lse_or_null, sparsed_pattern* out,
                                      float* scores_out_or_null, void* ws, size_t ws_bytes, void* cuda_stream) {
  Resolved rs;
  sparsed_status st = check_shape(shape, false, &rs);
  if (st != SPARSED_OK) return st;
  if (params == nullptr) return SPARSED_ERR_INVALID_ARG;
  if (params->block_size != 32 && params->block_size != 64 && params->block_size != 128) return SPARSED_ERR_UNSUPPORTED;
  if (shape->seq_len % params->block_size != 0) return SPARSED_ERR_ALIGNMENT;
  const int nb = shape->seq_len / params->block_size;
  int pb = 0, k_pre = 0, k_gen = 0;
  if ((st = kept_counts(params, nb, &pb, &k_pre, &k_gen)) != SPARSED_OK) return st;
  if (q == nullptr || k == nullptr) return SPARSED_ERR_INVALID_ARG;
  if (!aligned16(q) || !aligned16(k) || !aligned16(lse_or_null) || !aligned16(scores_out_or_null))
    return SPARSED_ERR_ALIGNMENT;
  if ((st = prepare_pattern(out, shape->batch, shape->heads_q, nb, params->block_size, k_pre + k_gen)) != SPARSED_OK)
    return st;
  // With few enough blocks per row the pooled-scoring kernel ranks each block-row in its own
  // tail; A' then goes to memory only if the caller asked for it.
  const bool fused = score_ranks_in_kernel(nb, params->block_size);
  // Up to 512 key blocks per row it also needs no log-sum-exp pass before it (one exponential per logit instead of two).
  const bool one_pass = lse_or_null == nullptr && score_in_one_pass(nb);
  const size_t bh = static_cast<size_t>(shape->batch) * shape->heads_q;
  const size_t score_bytes = round_up(bh * nb * nb * 4, 256);
  const size_t lse_bytes = round_up(bh * static_cast<size_t>(shape->seq_len) * 4, 256);
  // Workspace: room for A' wherever the ranking has a kernel of its own, and, as callers have always been asked for it
  // there, with 32-key blocks and beyond 1024 blocks per row; room for the LSE unless the caller has it.
  const bool need_score_ws = (!fused || nb > 1024 || params->block_size == 32) && scores_out_or_null == nullptr;
  const size_t required = SPARSED_STATUS_BYTES + (need_score_ws ? score_bytes : 0) + (lse_or_null ? 0 : lse_bytes);
  if ((st = check_ws(ws, ws_bytes, required)) != SPARSED_OK) return st;
  if ((st = check_arch()) != SPARSED_OK) return st;
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  uint8_t* base = static_cast<uint8_t*>(ws);
  float* scores = scores_out_or_null;
  size_t off = SPARSED_STATUS_BYTES;
  if (need_score_ws) {
    scores = reinterpret_cast<float*>(base + off);
    off += score_bytes;
  }
  CUtensorMap tq, tk;
  if ((st = make_tensor_map(&tq, q, shape->batch, shape->heads_q, shape->seq_len, rs.q, 128)) != SPARSED_OK) return st;
  if ((st = make_tensor_map(&tk, k, shape->batch, shape->heads_kv, shape->seq_len, rs.k, 64)) != SPARSED_OK) return st;
  ScoreParams sp;
  sp.scores = fused ? scores_out_or_null : scores;
  sp.lse = lse_or_null;
  sp.seq_len = shape->seq_len;
  sp.heads_q = shape->heads_q;
  sp.group = shape->heads_q / shape->heads_kv;
  sp.block_size = params->block_size;
  sp.scale_log2 = rs.scale_log2;
  sp.status = static_cast<DeviceStatus*>(ws);
  sp.row_ptr = fused ? out->row_ptr : nullptr;
  sp.col_idx = fused ? out->col_idx : nullptr;
  sp.pb = pb;
  sp.k_pre = k_pre;
  sp.k_gen = k_gen;
  sp.max_ctas = attn_max_ctas();
  sp.lse_out = nullptr;
  if (lse_or_null == nullptr && !one_pass) {
    sp.lse_out = reinterpret_cast<float*>(base + off);
    cudaError_t e = launch_row_stats(tq, tk, sp, shape->batch, stream);
    if (e != cudaSuccess) return cuda_fail(e);
    sp.lse = sp.lse_out;
  }
  cudaError_t e = launch_pooled_scores(tq, tk, sp, shape->batch, stream);
  if (e != cudaSuccess) return cuda_fail(e);
  if (fused) return SPARSED_OK;
  return run_topk(scores, shape->batch, shape->heads_q, nb, params->block_size, pb, k_pre, k_gen, out, stream);
}

sparsed_status sparsed_attention_step(const sparsed_shape* shape, const sparsed_select_params* params,
                                      int32_t step_1based, int32_t total_steps, double skip, const void* q,
                                      const void* k, const void* v, void* o, sparsed_pattern* pattern, void* ws,
                                      size_t ws_bytes, void* cuda_stream, int32_t* mode_out_or_null) {
  const int32_t mode = sparsed_schedule_mode(step_1based, total_steps, skip);
  if (mode < 0) return SPARSED_ERR_INVALID_ARG;
  if (mode_out_or_null != nullptr) *mode_out_or_null = mode;
  if (mode == SPARSED_MODE_FULL) return sparsed_attn_full(shape, q, k, v, o, nullptr, ws, ws_bytes, cuda_stream);
  if (mode == SPARSED_MODE_SPARSE) return sparsed_attn_sparse(shape, pattern, q, k, v, o, ws, ws_bytes, cuda_stream);
  // the switch step
  if (shape == nullptr || params == nullptr) return SPARSED_ERR_INVALID_ARG;
  size_t need = 0;
  sparsed_status st = sparsed_workspace_bytes(SPARSED_OP_ATTENTION_STEP, shape, params, &need);
  if (st != SPARSED_OK) return st;
  if ((st = check_ws(ws, ws_bytes, need)) != SPARSED_OK) return st;
  const size_t bh = static_cast<size_t>(shape->batch) * shape->heads_q;
  const size_t lse_bytes = round_up(bh * static_cast<size_t>(shape->seq_len) * 4, 256);
  uint8_t* base = static_cast<uint8_t*>(ws);
  if (step_uses_stats(shape, params)) {
    float* lse = reinterpret_cast<float*>(base + SPARSED_STATUS_BYTES);
    float* stats = reinterpret_cast<float*>(base + SPARSED_STATUS_BYTES + lse_bytes);
    if ((st = sparsed_attn_full_stats(shape, params->block_size, q, k, v, o, lse, stats, ws, ws_bytes, cuda_stream)) != SPARSED_OK)
      return st;
    return sparsed_select_from_stats(shape, params, lse, stats, pattern, nullptr, ws, ws_bytes, cuda_stream);
  }
  // [status][A' scratch of sparsed_select_pattern][LSE of the full pass]
  const size_t nb = static_cast<size_t>(shape->seq_len / params->block_size);
  const size_t score_bytes = round_up(bh * nb * nb * 4, 256);
  float* lse = reinterpret_cast<float*>(base + SPARSED_STATUS_BYTES + score_bytes);
  if ((st = sparsed_attn_full(shape, q, k, v, o, lse, ws, ws_bytes, cuda_stream)) != SPARSED_OK) return st;
  return sparsed_select_pattern(shape, params, q, k, lse, pattern, nullptr, ws, SPARSED_STATUS_BYTES + score_bytes,
                                cuda_stream);
}

sparsed_status sparsed_attention_step_variant(const sparsed_shape* shape, const sparsed_select_params* params,
                                              int32_t variant, int32_t step_1based, int32_t total_steps, double skip,
                                              const void* q, const void* k, const void* v, void* o,
                                              sparsed_pattern* pattern, void* ws, size_t ws_bytes, void* cuda_stream,
                                              int32_t* mode_out_or_null) {
  if (params == nullptr) return SPARSED_ERR_INVALID_ARG;
  if ((variant & ~(SPARSED_VARIANT_NO_REUSE | SPARSED_VARIANT_NO_ISOLATION)) != 0) return SPARSED_ERR_INVALID_ARG;
  sparsed_select_params p2 = *params;
  if (variant & SPARSED_VARIANT_NO_ISOLATION) p2.prefill_len = 0;
  const int32_t mode = sparsed_schedule_mode(step_1based, total_steps, skip);
  if (mode < 0) return SPARSED_ERR_INVALID_ARG;
  if (mode == SPARSED_MODE_SPARSE && (variant & SPARSED_VARIANT_NO_REUSE)) {
    // "without Sparse Reusing": this step's own Q and K give this step's pattern (pooled scoring and
    // ranking), then the block-sparse attention runs on it
    if (mode_out_or_null != nullptr) *mode_out_or_null = mode;
    sparsed_status st = sparsed_select_pattern(shape, &p2, q, k, nullptr, pattern, nullptr, ws, ws_bytes, cuda_stream);
    if (st != SPARSED_OK) return st;
    return sparsed_attn_sparse(shape, pattern, q, k, v, o, ws, ws_bytes, cuda_stream);
  }
  return sparsed_attention_step(shape, &p2, step_1based, total_steps, skip, q, k, v, o, pattern, ws, ws_bytes,
                                cuda_stream, mode_out_or_null);
}

sparsed_status sparsed_build_window_pattern(int32_t batch, int32_t heads_q, int32_t num_blocks, int32_t block_size,
                                            int32_t sink_blocks, int32_t window_blocks, sparsed_pattern* out,
                                            void* cuda_stream) {
  if (batch < 1 || heads_q < 1 || num_blocks < 1 || sink_blocks < 0 || window_blocks < 1) return SPARSED_ERR_INVALID_ARG;
  if (block_size != 32 && block_size != 64 && block_size != 128) return SPARSED_ERR_UNSUPPORTED;
  if (num_blocks > 16384) return SPARSED_ERR_UNSUPPORTED;
  if (out == nullptr || out->row_ptr == nullptr || out->col_idx == nullptr) return SPARSED_ERR_PATTERN;
  if (!aligned4(out->row_ptr) || !aligned4(out->col_idx)) return SPARSED_ERR_ALIGNMENT;
  const int sink = sink_blocks < num_blocks ? sink_blocks : num_blocks;
  const int half = (window_blocks - 1) / 2;
  const int64_t per_head = window_pattern_nnz_per_head(num_blocks, sink, half);
  const int64_t bh = static_cast<int64_t>(batch) * heads_q;
  const int64_t nnz = per_head * bh;
  if (nnz >= INT32_MAX || bh * num_blocks >= INT32_MAX) return SPARSED_ERR_UNSUPPORTED;
  if (out->col_capacity < nnz) return SPARSED_ERR_PATTERN;
  cudaError_t e = launch_window_pattern(out->row_ptr, out->col_idx, static_cast<int>(bh), num_blocks, sink, half,
                                        static_cast<int>(per_head), static_cast<cudaStream_t>(cuda_stream));
  if (e != cudaSuccess) return cuda_fail(e);
  out->nnz = nnz;
  out->block_size = block_size;
  out->num_blocks = num_blocks;
  out->batch = batch;
  out->heads_q = heads_q;
  return SPARSED_OK;
}

sparsed_status sparsed_pattern_validate(const sparsed_pattern* pattern, void* ws, size_t ws_bytes, void* cuda_stream) {
  if (pattern == nullptr || pattern->row_ptr == nullptr || pattern->col_idx == nullptr) return SPARSED_ERR_PATTERN;
  if (pattern->batch < 1 || pattern->heads_q < 1 || pattern->num_blocks < 1) return SPARSED_ERR_PATTERN;
  if (!aligned4(pattern->row_ptr) || !aligned4(pattern->col_idx)) return SPARSED_ERR_ALIGNMENT;
  sparsed_status st = check_ws(ws, ws_bytes, SPARSED_STATUS_BYTES);
  if (st != SPARSED_OK) return st;
  const int64_t rows = static_cast<int64_t>(pattern->batch) * pattern->heads_q * pattern->num_blocks;
  if (rows >= INT32_MAX) return SPARSED_ERR_UNSUPPORTED;
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  int* flag = reinterpret_cast<int*>(static_cast<uint8_t*>(ws) + 16);
  cudaError_t e = cudaMemsetAsync(flag, 0, sizeof(int), stream);
  if (e != cudaSuccess) return cuda_fail(e);
  e = launch_pattern_validate(pattern->row_ptr, pattern->col_idx, static_cast<int>(rows), pattern->num_blocks,
                              pattern->col_capacity, flag, stream);
  if (e != cudaSuccess) return cuda_fail(e);
  int host_flag = 0;
  e = cudaMemcpyAsync(&host_flag, flag, sizeof(int), cudaMemcpyDeviceToHost, stream);
  if (e != cudaSuccess) return cuda_fail(e);
  e = cudaStreamSynchronize(stream);
  if (e != cudaSuccess) return cuda_fail(e);
  return host_flag == 0 ? SPARSED_OK : SPARSED_ERR_PATTERN;
}

sparsed_status sparsed_selftest_wait_timeout(void* ws, size_t ws_bytes, void* cuda_stream) {
  sparsed_status st = check_ws(ws, ws_bytes, SPARSED_STATUS_BYTES);
  if (st != SPARSED_OK) return st;
  if ((st = check_arch()) != SPARSED_OK) return st;
  cudaError_t e = launch_wait_timeout_selftest(static_cast<DeviceStatus*>(ws), 99, static_cast<cudaStream_t>(cuda_stream));
  return e == cudaSuccess ? SPARSED_OK : cuda_fail(e);
}

sparsed_status sparsed_last_device_status(void* ws, void* cuda_stream, int32_t* code, int32_t* where) {
  if (ws == nullptr) return SPARSED_ERR_WORKSPACE;
  if (!aligned4(ws)) return SPARSED_ERR_ALIGNMENT;
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  int32_t host[2] = {0, 0};
  cudaError_t e = cudaMemcpyAsync(host, ws, sizeof(host), cudaMemcpyDeviceToHost, stream);
  if (e != cudaSuccess) return cuda_fail(e);
  e = cudaStreamSynchronize(stream);
  if (e != cudaSuccess) return cuda_fail(e);
  if (code != nullptr) *code = host[0];
  if (where != nullptr) *where = host[1];
  return host[0] == 0 ? SPARSED_OK : SPARSED_ERR_DEVICE_TIMEOUT;
}

}  // extern "C"

// ------------------------------------------------------------------------------------------
// Packed sequences and the paged key-value cache
// ------------------------------------------------------------------------------------------
namespace {

// Strides of a [rows, heads, 128] tensor (row, head), all-zero = contiguous.
sparsed_status row_strides(const int64_t in[2], int heads, int64_t out[2]) {
  const bool given = in != nullptr && (in[0] != 0 || in[1] != 0);
  out[0] = given ? in[0] : static_cast<int64_t>(heads) * 128;
  out[1] = given ? in[1] : 128;
  if (out[0] <= 0 || out[1] <= 0) return SPARSED_ERR_INVALID_ARG;
  if (out[0] % 8 != 0 || out[1] % 8 != 0) return SPARSED_ERR_ALIGNMENT;
  if (out[0] < 128 || out[1] < 128) return SPARSED_ERR_INVALID_ARG;
  return SPARSED_OK;
}

sparsed_status check_scale(float scale, float* scale_log2) {
  if (!(scale >= 0.f) || !std::isfinite(scale)) return SPARSED_ERR_INVALID_ARG;
  *scale_log2 = (scale == 0.f ? 1.0f / std::sqrt(128.f) : scale) * 1.44269504088896341f;
  return SPARSED_OK;
}

// Whether a packed call runs on the CTA-pair kernel. SPARSED_PACKED_KERNEL=pair|single (read once) sends every call to one of the
// two, for measurements and tests.
bool packed_kernel_is_pair(const sparsed_packed* s, int pack, int tile_tokens) {
  static const int forced = [] {
    const char* v = std::getenv("SPARSED_PACKED_KERNEL");
    if (v != nullptr && std::strcmp(v, "pair") == 0) return 1;
    if (v != nullptr && std::strcmp(v, "single") == 0) return 0;
    return -1;
  }();
  if (forced >= 0) return forced == 1;
  return packed_pair_pays(s->num_seqs, s->total_q, s->total_k, s->heads_q / pack, tile_tokens, s->causal != 0);
}

// The sizes of a cache alone (what the workspace queries need).
sparsed_status check_cache_sizes(const sparsed_cache* c) {
  if (c == nullptr) return SPARSED_ERR_INVALID_ARG;
  if (c->num_pages < 1 || c->heads_kv < 1 || c->batch < 1 || c->max_pages < 1) return SPARSED_ERR_INVALID_ARG;
  if (c->head_dim != 128) return SPARSED_ERR_UNSUPPORTED;
  if (c->dtype != SPARSED_DTYPE_BF16 && c->dtype != SPARSED_DTYPE_FP16) return SPARSED_ERR_UNSUPPORTED;
  if (c->page_size < 16 || c->page_size > 256 || (c->page_size & (c->page_size - 1)) != 0) return SPARSED_ERR_UNSUPPORTED;
  // positions of a sequence, and (sequence, head) pairs, are counted in 32 bits
  if (static_cast<int64_t>(c->max_pages) * c->page_size > (INT32_MAX >> 1)) return SPARSED_ERR_UNSUPPORTED;
  if (static_cast<int64_t>(c->batch) * c->heads_kv > (INT32_MAX >> 5)) return SPARSED_ERR_UNSUPPORTED;
  return SPARSED_OK;
}

sparsed_status check_cache(const sparsed_cache* c, CacheView* view) {
  sparsed_status st = check_cache_sizes(c);
  if (st != SPARSED_OK) return st;
  if (c->k == nullptr || c->v == nullptr || c->page_table == nullptr || c->seq_lens == nullptr) return SPARSED_ERR_INVALID_ARG;
  if (!aligned16(c->k) || !aligned16(c->v) || !aligned4(c->page_table) || !aligned4(c->seq_lens)) return SPARSED_ERR_ALIGNMENT;
  view->k = static_cast<uint16_t*>(c->k);
  view->v = static_cast<uint16_t*>(c->v);
  view->table = c->page_table;
  view->lens = c->seq_lens;
  view->table_stride = c->table_stride == 0 ? c->max_pages : c->table_stride;
  if (view->table_stride < 0) return SPARSED_ERR_INVALID_ARG;
  const int64_t* given[2] = {c->k_strides, c->v_strides};
  int64_t* page[2] = {&view->k_page, &view->v_page};
  int64_t* place[2] = {&view->k_place, &view->v_place};
  int64_t* head[2] = {&view->k_head, &view->v_head};
  for (int i = 0; i < 2; ++i) {
    const int64_t* s = given[i];
    const bool contiguous = s[0] == 0 && s[1] == 0 && s[2] == 0;
    *head[i] = contiguous ? 128 : s[2];
    *place[i] = contiguous ? 128ll * c->heads_kv : s[1];
    *page[i] = contiguous ? 128ll * c->heads_kv * c->page_size : s[0];
    const int64_t all[3] = {*page[i], *place[i], *head[i]};
    for (int64_t x : all) {
      if (x < 128) return SPARSED_ERR_INVALID_ARG;
      if (x % 8 != 0) return SPARSED_ERR_ALIGNMENT;
    }
  }
  view->num_pages = c->num_pages;
  view->page_shift = 0;
  while ((1 << view->page_shift) < c->page_size) ++view->page_shift;
  view->heads_kv = c->heads_kv;
  view->batch = c->batch;
  view->max_pages = c->max_pages;
  return SPARSED_OK;
}

}  // namespace

extern "C" sparsed_status sparsed_attn_packed(const sparsed_packed* shape, const int32_t* cu_q, const int32_t* cu_k,
                                              const void* q, const void* k, const void* v, void* o, float* lse_or_null,
                                              void* ws, size_t ws_bytes, void* cuda_stream) {
  if (shape == nullptr) return SPARSED_ERR_INVALID_ARG;
  if (shape->num_seqs < 0 || shape->total_q < 0 || shape->total_k < 0 || shape->heads_q < 1 || shape->heads_kv < 1)
    return SPARSED_ERR_INVALID_ARG;
  if (shape->heads_q % shape->heads_kv != 0) return SPARSED_ERR_INVALID_ARG;
  if (shape->causal != 0 && shape->causal != 1) return SPARSED_ERR_INVALID_ARG;
  if (shape->head_dim != 128) return SPARSED_ERR_UNSUPPORTED;
  if (shape->dtype != SPARSED_DTYPE_BF16 && shape->dtype != SPARSED_DTYPE_FP16) return SPARSED_ERR_UNSUPPORTED;
  PackedParams p;
  int64_t qs[2], ks[2], vs[2], os[2];
  sparsed_status st;
  if ((st = check_scale(shape->softmax_scale, &p.scale_log2)) != SPARSED_OK) return st;
  if ((st = row_strides(shape->q_strides, shape->heads_q, qs)) != SPARSED_OK) return st;
  if ((st = row_strides(shape->k_strides, shape->heads_kv, ks)) != SPARSED_OK) return st;
  if ((st = row_strides(shape->v_strides, shape->heads_kv, vs)) != SPARSED_OK) return st;
  if ((st = row_strides(shape->o_strides, shape->heads_q, os)) != SPARSED_OK) return st;
  p.group = shape->heads_q / shape->heads_kv;
  p.pack = packed_heads_per_tile(p.group);
  p.tile_tokens = 128 / p.pack;
  const bool pair = packed_kernel_is_pair(shape, p.pack, p.tile_tokens);
  const int64_t tiles = static_cast<int64_t>(shape->total_q) / (pair ? 4 * p.tile_tokens : p.tile_tokens) + shape->num_seqs;
  if (tiles * (shape->heads_q / p.pack) > INT32_MAX / 2) return SPARSED_ERR_UNSUPPORTED;
  const bool nothing = shape->num_seqs == 0 || shape->total_q == 0, no_keys = shape->total_k == 0;
  if (cu_q == nullptr || cu_k == nullptr) return SPARSED_ERR_INVALID_ARG;
  if (!nothing && (q == nullptr || o == nullptr)) return SPARSED_ERR_INVALID_ARG;
  if (!nothing && !no_keys && (k == nullptr || v == nullptr)) return SPARSED_ERR_INVALID_ARG;
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(o) || !aligned4(cu_q) || !aligned4(cu_k) ||
      !aligned4(lse_or_null))
    return SPARSED_ERR_ALIGNMENT;
  if ((st = check_ws(ws, ws_bytes, SPARSED_STATUS_BYTES)) != SPARSED_OK) return st;
  if (nothing) return SPARSED_OK;
  if ((st = check_arch()) != SPARSED_OK) return st;
  CUtensorMap tq, tk, tv;
  if ((st = make_packed_query_map(&tq, q, shape->total_q, shape->heads_kv, p.group, qs[0], qs[1], p.pack, p.tile_tokens)) != SPARSED_OK)
    return st;
  if (no_keys) {
    tk = tv = tq;   // (nothing is loaded through them)
  } else {
    if ((st = make_packed_key_map(&tk, k, shape->total_k, shape->heads_kv, ks, pair ? 32 : 64)) != SPARSED_OK) return st;
    if ((st = make_packed_key_map(&tv, v, shape->total_k, shape->heads_kv, vs, 64)) != SPARSED_OK) return st;
  }
  p.cu_q = cu_q;
  p.cu_k = cu_k;
  p.o = o;
  p.o_stride_t = os[0];
  p.o_stride_h = os[1];
  p.v = v;
  p.v_stride_t = vs[0];
  p.v_stride_h = vs[1];
  p.lse = lse_or_null;
  p.num_seqs = shape->num_seqs;
  p.total_q = shape->total_q;
  p.total_k = shape->total_k;
  p.heads_q = shape->heads_q;
  p.causal = shape->causal;
  p.tiles = static_cast<int>(tiles);
  // key-value heads whose K and V (512 bytes a key) take 48 MB of the L2 together, one at least
  const int64_t heads_in_l2 = (int64_t{48} << 20) / (512ll * (shape->total_k > 0 ? shape->total_k : 1));
  const int64_t heads_at_once = heads_in_l2 >= shape->heads_kv ? shape->heads_kv : (heads_in_l2 > 1 ? heads_in_l2 : 1);
  p.heads_per_pass = static_cast<int>(heads_at_once * (p.group / p.pack));
  p.max_ctas = attn_max_ctas();
  p.slow_path_events = reinterpret_cast<unsigned long long*>(static_cast<uint8_t*>(ws) + 32);
  p.status = static_cast<DeviceStatus*>(ws);
  auto launch = pair ? launch_attn_packed_pair : launch_attn_packed;
  cudaError_t e = launch(tq, tk, tv, p, shape->dtype == SPARSED_DTYPE_FP16, static_cast<cudaStream_t>(cuda_stream));
  return e == cudaSuccess ? SPARSED_OK : cuda_fail(e);
}

extern "C" sparsed_status sparsed_cache_write(const sparsed_cache* cache, const void* k_new, const int64_t k_new_strides[2],
                                              const void* v_new, const int64_t v_new_strides[2], const int32_t* cu_new,
                                              int32_t total_new, void* ws, size_t ws_bytes, void* cuda_stream) {
  CacheWriteParams p;
  sparsed_status st = check_cache(cache, &p.cache);
  if (st != SPARSED_OK) return st;
  if (total_new < 0 || cu_new == nullptr) return SPARSED_ERR_INVALID_ARG;
  int64_t ks[2], vs[2];
  if ((st = row_strides(k_new_strides, cache->heads_kv, ks)) != SPARSED_OK) return st;
  if ((st = row_strides(v_new_strides, cache->heads_kv, vs)) != SPARSED_OK) return st;
  if (total_new > 0 && (k_new == nullptr || v_new == nullptr)) return SPARSED_ERR_INVALID_ARG;
  if (!aligned16(k_new) || !aligned16(v_new) || !aligned4(cu_new)) return SPARSED_ERR_ALIGNMENT;
  if ((st = check_ws(ws, ws_bytes, SPARSED_STATUS_BYTES)) != SPARSED_OK) return st;
  if (total_new == 0) return SPARSED_OK;
  if ((st = check_arch()) != SPARSED_OK) return st;
  p.k = static_cast<const uint16_t*>(k_new);
  p.v = static_cast<const uint16_t*>(v_new);
  p.k_token = ks[0];
  p.k_head = ks[1];
  p.v_token = vs[0];
  p.v_head = vs[1];
  p.cu = cu_new;
  p.total = total_new;
  p.tokens_at_once = p.tokens_per_warp = 1;
  p.status = static_cast<DeviceStatus*>(ws);
  cudaError_t e = launch_cache_write(p, static_cast<cudaStream_t>(cuda_stream));
  return e == cudaSuccess ? SPARSED_OK : cuda_fail(e);
}

// Whether two arrays of 4-byte elements share any.
static bool overlap(const void* a, int64_t n_a, const void* b, int64_t n_b) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y ? y - x < static_cast<uintptr_t>(n_a) * 4 : x - y < static_cast<uintptr_t>(n_b) * 4;
}

// The sizes of a paged call: query heads, and units of work that are counted in 32 bits.
static sparsed_status check_paged_sizes(const sparsed_cache* cache, int32_t heads_q) {
  sparsed_status st = check_cache_sizes(cache);
  if (st != SPARSED_OK) return st;
  if (heads_q < 1 || heads_q % cache->heads_kv != 0) return SPARSED_ERR_INVALID_ARG;
  const int64_t keys = static_cast<int64_t>(cache->max_pages) * cache->page_size;
  if (static_cast<int64_t>(cache->batch) * heads_q * (keys / 64 + 1) > INT32_MAX / 2) return SPARSED_ERR_UNSUPPORTED;
  if (heads_q / cache->heads_kv > 4096) return SPARSED_ERR_UNSUPPORTED;   // (their LSE lie in shared memory, 16 KB)
  return SPARSED_OK;
}

extern "C" sparsed_status sparsed_paged_workspace_bytes(const sparsed_cache* cache, int32_t heads_q, int32_t with_mass,
                                                        size_t* out_bytes) {
  if (out_bytes == nullptr) return SPARSED_ERR_INVALID_ARG;
  sparsed_status st = check_paged_sizes(cache, heads_q);
  if (st != SPARSED_OK) return st;
  *out_bytes = static_cast<size_t>(paged_layout(cache->batch, cache->heads_kv, heads_q / cache->heads_kv, cache->max_pages,
                                                cache->page_size, with_mass != 0).bytes);
  return SPARSED_OK;
}

extern "C" sparsed_status sparsed_attn_paged(const sparsed_cache* cache, int32_t heads_q, const void* q,
                                             const int64_t q_strides[2], void* o, const int64_t o_strides[2],
                                             float softmax_scale, float* lse_or_null, const float* mass_in_or_null,
                                             float* mass_out_or_null, int64_t mass_capacity, void* ws, size_t ws_bytes,
                                             void* cuda_stream) {
  PagedParams p;
  sparsed_status st = check_paged_sizes(cache, heads_q);
  if (st != SPARSED_OK) return st;
  if ((st = check_cache(cache, &p.cache)) != SPARSED_OK) return st;
  if ((st = check_scale(softmax_scale, &p.scale_log2)) != SPARSED_OK) return st;
  int64_t qs[2], os[2];
  if ((st = row_strides(q_strides, heads_q, qs)) != SPARSED_OK) return st;
  if ((st = row_strides(o_strides, heads_q, os)) != SPARSED_OK) return st;
  if (q == nullptr || o == nullptr) return SPARSED_ERR_INVALID_ARG;
  const bool with_mass = mass_out_or_null != nullptr;
  if (!with_mass && mass_in_or_null != nullptr) return SPARSED_ERR_INVALID_ARG;
  if (with_mass && mass_capacity < static_cast<int64_t>(cache->max_pages) * cache->page_size) return SPARSED_ERR_INVALID_ARG;
  if (!aligned16(q) || !aligned16(o) || !aligned4(lse_or_null) || !aligned4(mass_in_or_null) || !aligned4(mass_out_or_null))
    return SPARSED_ERR_ALIGNMENT;
  // (each weight is read by the thread that writes it, in no order: the same array or another)
  const int64_t masses = static_cast<int64_t>(cache->batch) * cache->heads_kv * mass_capacity;
  if (mass_in_or_null != nullptr && mass_in_or_null != mass_out_or_null && overlap(mass_in_or_null, masses, mass_out_or_null, masses))
    return SPARSED_ERR_INVALID_ARG;
  const int group = heads_q / cache->heads_kv;
  const PagedLayout at = paged_layout(cache->batch, cache->heads_kv, group, cache->max_pages, cache->page_size, with_mass);
  if ((st = check_ws(ws, ws_bytes, static_cast<size_t>(at.bytes))) != SPARSED_OK) return st;
  if ((st = check_arch()) != SPARSED_OK) return st;
  uint8_t* base = static_cast<uint8_t*>(ws);
  p.q = static_cast<const uint16_t*>(q);
  p.o = static_cast<uint16_t*>(o);
  p.q_seq = qs[0];
  p.q_head = qs[1];
  p.o_seq = os[0];
  p.o_head = os[1];
  p.lse = lse_or_null;
  p.mass_in = mass_in_or_null;
  p.mass_out = mass_out_or_null;
  p.mass_capacity = mass_capacity;
  p.group = group;
  p.ctas = p.fills = 0;   // (launch_attn_paged)
  p.prefix = reinterpret_cast<int32_t*>(base + at.prefix);
  p.lse2 = reinterpret_cast<float*>(base + at.lse2);
  p.part_ml = reinterpret_cast<float2*>(base + at.part_ml);
  p.part_o = reinterpret_cast<float*>(base + at.part_o);
  p.logits = with_mass ? reinterpret_cast<float*>(base + at.logits) : nullptr;
  p.status = static_cast<DeviceStatus*>(ws);
  CUtensorMap tk, tv;
  const CacheView& c = p.cache;
  if ((st = make_pool_map(&tk, c.k, c.num_pages, cache->page_size, c.heads_kv, c.k_page, c.k_place, c.k_head)) != SPARSED_OK) return st;
  if ((st = make_pool_map(&tv, c.v, c.num_pages, cache->page_size, c.heads_kv, c.v_page, c.v_place, c.v_head)) != SPARSED_OK) return st;
  cudaError_t e = launch_attn_paged(tk, tv, p, attn_max_ctas() / 2, cache->dtype == SPARSED_DTYPE_FP16, static_cast<cudaStream_t>(cuda_stream));
  return e == cudaSuccess ? SPARSED_OK : cuda_fail(e);
}

extern "C" sparsed_status sparsed_evict_workspace_bytes(const sparsed_cache* from, size_t* out_bytes) {
  if (out_bytes == nullptr) return SPARSED_ERR_INVALID_ARG;
  sparsed_status st = check_cache_sizes(from);
  if (st != SPARSED_OK) return st;
  *out_bytes = SPARSED_STATUS_BYTES;
  return SPARSED_OK;
}

extern "C" sparsed_status sparsed_cache_evict(const sparsed_cache* from, const float* mass, int64_t mass_capacity, int32_t keep,
                                              int32_t recent, const sparsed_cache* to, float* mass_out,
                                              int64_t mass_out_capacity, int32_t* kept, void* ws, size_t ws_bytes,
                                              void* cuda_stream) {
  EvictParams p;
  sparsed_status st = check_cache(from, &p.from);
  if (st != SPARSED_OK) return st;
  if ((st = check_cache(to, &p.to)) != SPARSED_OK) return st;
  if (from->batch != to->batch || from->heads_kv != to->heads_kv || from->dtype != to->dtype) return SPARSED_ERR_INVALID_ARG;
  if (overlap(from->seq_lens, from->batch, to->seq_lens, to->batch)) return SPARSED_ERR_INVALID_ARG;   // (read by many CTAs while it is written)
  if (mass == nullptr || mass_out == nullptr || kept == nullptr) return SPARSED_ERR_INVALID_ARG;
  if (keep < 1 || recent < 0 || recent > keep) return SPARSED_ERR_INVALID_ARG;
  // a row has no more keys than its cache has places, whatever `keep` allows (and the places are few enough for 32 bits)
  const int64_t room = static_cast<int64_t>(from->max_pages) * from->page_size, most = keep < room ? keep : room;
  if (most > static_cast<int64_t>(to->max_pages) * to->page_size) return SPARSED_ERR_INVALID_ARG;
  if (mass_capacity < room || mass_out_capacity < most) return SPARSED_ERR_INVALID_ARG;
  if (keep > (INT32_MAX >> 1)) return SPARSED_ERR_UNSUPPORTED;   // as the places of a cache
  const int64_t rows = static_cast<int64_t>(from->batch) * from->heads_kv;
  if (rows * (keep / 8 + 1ll) > INT32_MAX / 2) return SPARSED_ERR_UNSUPPORTED;
  if (!aligned4(mass) || !aligned4(mass_out) || !aligned4(kept)) return SPARSED_ERR_ALIGNMENT;
  if ((st = check_ws(ws, ws_bytes, SPARSED_STATUS_BYTES)) != SPARSED_OK) return st;
  if (overlap(mass, rows * mass_capacity, mass_out, rows * mass_out_capacity)) return SPARSED_ERR_INVALID_ARG;
  if ((st = check_arch()) != SPARSED_OK) return st;
  p.mass = mass;
  p.mass_out = mass_out;
  p.mass_capacity = mass_capacity;
  p.mass_out_capacity = mass_out_capacity;
  p.kept = kept;
  p.keep = keep;
  p.recent = recent;
  p.status = static_cast<DeviceStatus*>(ws);
  cudaError_t e = launch_cache_evict(p, static_cast<cudaStream_t>(cuda_stream));
  return e == cudaSuccess ? SPARSED_OK : cuda_fail(e);
}

// ------------------------------------------------------------------------------------------
// Selection without a caller workspace: the scratch lives in this library's device image.
// ------------------------------------------------------------------------------------------
namespace {

constexpr size_t kStaticScratchBytes = SPARSED_STATIC_SCRATCH_BYTES;

// Scratch for sparsed_select_pattern_static: status block, pooled scores A', and the LSE
// rows when the caller has none. One copy per GPU that loads the library, held until exit.
static __device__ __align__(256) unsigned char g_select_scratch[kStaticScratchBytes];

std::mutex g_scratch_mutex;
void* g_scratch_addr[64] = {};

// In host code `g_select_scratch` is only a handle for the runtime, not a device address:
// the address a kernel may use is looked up once per device with that device current.
sparsed_status static_scratch_address(void** out) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return cuda_fail(e);
  if (dev < 0 || dev >= 64) return SPARSED_ERR_UNSUPPORTED;
  std::lock_guard<std::mutex> lock(g_scratch_mutex);
  if (g_scratch_addr[dev] == nullptr) {
    void* ptr = nullptr;
    e = cudaGetSymbolAddress(&ptr, g_select_scratch);
    if (e != cudaSuccess) return cuda_fail(e);
    if (ptr == nullptr) return cuda_fail(cudaErrorInvalidSymbol);
    g_scratch_addr[dev] = ptr;
  }
  *out = g_scratch_addr[dev];
  return SPARSED_OK;
}

}  // namespace

extern "C" sparsed_status sparsed_select_pattern_static(const sparsed_shape* shape,
                                                        const sparsed_select_params* params, const void* q,
                                                        const void* k, const float* lse_or_null,
                                                        sparsed_pattern* out, void* cuda_stream) {
  if (shape == nullptr || params == nullptr) return SPARSED_ERR_INVALID_ARG;
  // Size check first, on the host, so that an oversized request never reaches the device.
  size_t full = 0;
  sparsed_status st = sparsed_workspace_bytes(SPARSED_OP_SELECT_PATTERN, shape, params, &full);
  if (st != SPARSED_OK) return st;
  const size_t bh = static_cast<size_t>(shape->batch) * static_cast<size_t>(shape->heads_q);
  const size_t lse_bytes = round_up(bh * static_cast<size_t>(shape->seq_len) * 4, 256);
  const size_t needed = full - (lse_or_null != nullptr ? lse_bytes : 0);
  if (needed > kStaticScratchBytes) return SPARSED_ERR_WORKSPACE;
  void* scratch = nullptr;
  if ((st = static_scratch_address(&scratch)) != SPARSED_OK) return st;
  // The array keeps whatever the previous call left: the status block must start at zero;
  // scores and LSE rows are fully rewritten by the kernels before anything reads them.
  cudaError_t e = cudaMemsetAsync(scratch, 0, SPARSED_STATUS_BYTES, static_cast<cudaStream_t>(cuda_stream));
  if (e != cudaSuccess) return cuda_fail(e);
  return sparsed_select_pattern(shape, params, q, k, lse_or_null, out, nullptr, scratch, kStaticScratchBytes,
                                cuda_stream);
}

