// C ABI of attention with shaped scores, of the packed cache and of eviction:
// argument checks on the host, then the launches.
#include <algorithm>

#include "api_checks.h"
#include "packed.h"
#include "shaped.h"
#include "shaped_ops.h"

namespace {

using namespace neo;

constexpr float kLog2e = 1.4426950408889634f;
static_assert(kPackedRecord == NEO_PACKED_RECORD_BYTES, "record size");

// Sizes that every call has.
neo_status check_sizes(int32_t batch, int32_t mbps, int32_t hkv, int32_t head_dim,
                       int32_t block_size, int32_t num_blocks) {
  if (batch < 0) return set_error(NEO_ERR_INVALID_ARG, "batch (%d) is negative", batch);
  if (hkv <= 0) return set_error(NEO_ERR_INVALID_ARG, "num_kv_heads (%d) must be positive", hkv);
  if (head_dim != kHeadDim || block_size != kBlock)
    return set_error(NEO_ERR_UNSUPPORTED, "head_dim %d / block_size %d unsupported (128 / 16)",
                     head_dim, block_size);
  if (batch == 0) return NEO_OK;
  if (mbps <= 0 || num_blocks <= 0)
    return set_error(NEO_ERR_INVALID_ARG,
                     "max_blocks_per_seq (%d) and num_blocks (%d) must be positive", mbps,
                     num_blocks);
  if ((int64_t)mbps * kBlock >= ((int64_t)1 << 31) - 512)
    return set_error(NEO_ERR_INVALID_ARG, "max_blocks_per_seq too large");
  if ((int64_t)batch * (mbps + kPairCostLong) > (((int64_t)1 << 31) - 1) / hkv)
    return set_error(NEO_ERR_INVALID_ARG,
                     "batch * (max_blocks_per_seq + %d) * num_kv_heads must stay below 2^31",
                     kPairCostLong);
  return NEO_OK;
}

// The stride of a bf16 cache's blocks, in bytes.
neo_status bf16_stride(int64_t stride, int32_t hkv, int32_t num_blocks, int64_t* bytes) {
  int64_t elems = 0;
  neo_status st = check_block_stride(stride, (int64_t)hkv * kTileElems, "kv_block_stride", &elems);
  if (st == NEO_OK) st = check_span(elems, num_blocks, "kv_block_stride");
  *bytes = 2 * elems;
  return st;
}

// The stride of a packed cache's blocks, in bytes: 0 for dense.
neo_status packed_stride(int64_t stride, int32_t hkv, int32_t num_blocks, int64_t* bytes) {
  const int64_t dense = (int64_t)hkv * kPackedRecord;
  if (stride != 0 && (stride < dense || stride % 16 != 0 || stride > ((int64_t)1 << 40)))
    return set_error(NEO_ERR_INVALID_ARG,
                     "block_stride %lld must be 0 or a multiple of 16 of at least %lld bytes "
                     "(and at most 2^40)",
                     (long long)stride, (long long)dense);
  *bytes = stride != 0 ? stride : dense;
  return check_span(*bytes, num_blocks, "block_stride");
}

neo_status check_ints(const void* p, const char* name, bool may_be_null = false) {
  if (!p && !may_be_null) return set_error(NEO_ERR_INVALID_ARG, "%s is NULL", name);
  if (!aligned(p, 4)) return set_error(NEO_ERR_INVALID_ARG, "%s must be 4-byte aligned", name);
  return NEO_OK;
}
neo_status check_words(const void* p, const char* name) {
  if (!p) return set_error(NEO_ERR_INVALID_ARG, "%s is NULL", name);
  if (!aligned(p, 16)) return set_error(NEO_ERR_INVALID_ARG, "%s must be 16-byte aligned", name);
  return NEO_OK;
}

#define NEO_TRY(expr)                          \
  do {                                         \
    const neo_status try_status = (expr);      \
    if (try_status != NEO_OK) return try_status; \
  } while (0)

// The scores' part of a call: heads, scale and shape into *p.
neo_status set_scores(ShapedParams* p, int32_t hq, int32_t hkv, int32_t head_dim, float scale,
                      const neo_score_shape* shape) {
  NEO_TRY(check_heads(hq, hkv, head_dim));
  if (!isfinite(scale)) return set_error(NEO_ERR_INVALID_ARG, "scale is not finite");
  const float cap = shape ? shape->softcap : 0.f;
  if (!(cap >= 0.f) || !isfinite(cap * kLog2e))
    return set_error(NEO_ERR_INVALID_ARG, "softcap must be 0 (none) or positive and finite");
  if (cap > 0.f && !isfinite(scale / cap))
    return set_error(NEO_ERR_INVALID_ARG, "scale / softcap is not finite");
  p->hq = hq;
  p->hkv = hkv;
  p->scale_log2 = scale * kLog2e;
  p->cap_in = cap > 0.f ? scale / cap : 0.f;
  p->cap_log2 = cap * kLog2e;
  p->slopes = shape ? shape->slopes : nullptr;
  p->starts = shape ? shape->starts : nullptr;
  p->prefix = shape ? shape->prefix_lens : nullptr;
  NEO_TRY(check_ints(p->slopes, "slopes", true));
  NEO_TRY(check_ints(p->starts, "starts", true));
  return check_ints(p->prefix, "prefix_lens", true);
}

// Workgroups of a (request, kv head) pair: as many as fill the compute units once,
// at most one for every 16 steps of the longest request the table holds.
int32_t parts_of(int32_t batch, int32_t hkv, int32_t mbps, int32_t blocks_per_step, int32_t cus) {
  const int64_t pairs = (int64_t)batch * hkv;
  const int32_t most = (mbps - 1) / (16 * blocks_per_step) + 1;
  return (int32_t)std::min<int64_t>(most, std::max<int64_t>(1, cus / pairs));
}

// Compute units that an attention call is cut for, at most. Of the workspace's
// NEO_MAX_SLICES counters and slots it uses a counter per pair or workgroup, and a slot per
// share (one and a half for every compute unit) or two per workgroup of slices.
constexpr int32_t kMostGroups = NEO_MAX_SLICES / 16;

struct Cache {
  const void* k;
  const void* v;   // null: packed
  int64_t stride;  // as the caller gave it
};

neo_status set_cache(ShapedParams* p, const Cache& c, bool packed, bool want_v,
                     const int32_t* table, const int32_t* lens, int32_t batch, int32_t mbps,
                     int32_t num_blocks) {
  NEO_TRY(packed ? packed_stride(c.stride, p->hkv, num_blocks, &p->blk_bytes)
                 : bf16_stride(c.stride, p->hkv, num_blocks, &p->blk_bytes));
  NEO_TRY(check_words(c.k, packed ? "cache" : "k_cache"));
  if (!packed && want_v) NEO_TRY(check_words(c.v, "v_cache"));
  NEO_TRY(check_ints(table, "block_table"));
  NEO_TRY(check_ints(lens, "seq_lens"));
  p->k = static_cast<const uint8_t*>(c.k);
  p->v = static_cast<const uint8_t*>(c.v);
  p->table = table;
  p->lens = lens;
  p->batch = batch;
  p->mbps = mbps;
  p->num_blocks = num_blocks;
  return NEO_OK;
}

neo_status launched(hipError_t e, const char* what) {
  if (e != hipSuccess) return set_error(NEO_ERR_HIP, "%s launch: %s", what, hipGetErrorString(e));
  return ok();
}

neo_status attend(const void* q, const Cache& cache, bool packed, const int32_t* table,
                  const int32_t* lens, int32_t hq, int32_t hkv, int32_t head_dim,
                  int32_t block_size, float scale, const neo_score_shape* shape, float* out,
                  float* lse, int32_t batch, int32_t mbps, int32_t num_blocks, void* workspace,
                  size_t workspace_bytes, void* stream) {
  ShapedParams p = {};
  NEO_TRY(set_scores(&p, hq, hkv, head_dim, scale, shape));
  NEO_TRY(check_sizes(batch, mbps, hkv, head_dim, block_size, num_blocks));
  if (batch == 0) return ok();
  NEO_TRY(set_cache(&p, cache, packed, true, table, lens, batch, mbps, num_blocks));
  NEO_TRY(check_words(q, "q"));
  NEO_TRY(check_words(out, "out"));
  NEO_TRY(check_ints(lse, "lse", true));
  const int32_t group = hq / hkv;
  const WorkspaceLayout wl = workspace_layout(batch, group);
  if (!workspace || workspace_bytes < wl.total)
    return set_error(NEO_ERR_WORKSPACE, "workspace needs %zu bytes, got %zu", wl.total,
                     workspace ? workspace_bytes : (size_t)0);
  if (!aligned(workspace, 256))
    return set_error(NEO_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
  int32_t cus = 0, xcds = 0;
  NEO_TRY(device_shape(&cus, &xcds));
  char* ws = static_cast<char*>(workspace);
  p.q = static_cast<const uint16_t*>(q);
  p.out = out;
  p.lse = lse;
  p.counters = reinterpret_cast<int32_t*>(ws + wl.counters);
  p.part_ml = reinterpret_cast<float*>(ws + wl.part_lse);
  p.part_o = reinterpret_cast<float*>(ws + wl.part_o);
  // In slices where there are more pairs than compute units, in pairs or shares of them
  // otherwise. Both ways, at 8 to 256 pairs shares are faster by 2 to 10 us (64 pairs of
  // 2048 tokens 17 us, in slices 22); at 512 they are even; slices gain from there on:
  // packed, 1024 pairs of 256 to 4096 tokens 69 instead of 79 us, 4096 pairs 223 instead of
  // 275 us.
  cus = std::min(cus, kMostGroups);
  p.parts = parts_of(batch, hkv, mbps, packed ? 4 : 1, cus);
  p.spare = std::max(1, cus / 2);
  p.slices = (int64_t)batch * hkv > cus ? cus : 0;
  hipStream_t s = static_cast<hipStream_t>(stream);
  return launched(packed ? launch_shaped_packed(p, group, false, s)
                         : launch_shaped_bf16(p, group, false, s),
                  "attention");
}

neo_status add_weights(const float* sums, float* sums_out, int64_t sums_stride, const float* lse,
                       const void* q, const Cache& cache, bool packed, const int32_t* table,
                       const int32_t* lens, int32_t hq, int32_t hkv, int32_t head_dim,
                       int32_t block_size, float scale, const neo_score_shape* shape,
                       int32_t batch, int32_t mbps, int32_t num_blocks, void* stream) {
  ShapedParams p = {};
  NEO_TRY(set_scores(&p, hq, hkv, head_dim, scale, shape));
  NEO_TRY(check_sizes(batch, mbps, hkv, head_dim, block_size, num_blocks));
  if (batch == 0) return ok();
  NEO_TRY(set_cache(&p, cache, packed, false, table, lens, batch, mbps, num_blocks));
  NEO_TRY(check_words(q, "q"));
  NEO_TRY(check_ints(sums, "sums"));
  NEO_TRY(check_ints(sums_out, "sums_out"));
  NEO_TRY(check_ints(lse, "lse"));
  if (sums_stride < (int64_t)mbps * kBlock)
    return set_error(NEO_ERR_INVALID_ARG,
                     "sums_stride (%lld) must be at least max_blocks_per_seq * block_size",
                     (long long)sums_stride);
  int32_t cus = 0, xcds = 0;
  NEO_TRY(device_shape(&cus, &xcds));
  p.q = static_cast<const uint16_t*>(q);
  p.sums = sums;
  p.sums_out = sums_out;
  p.sums_stride = sums_stride;
  p.lse_in = lse;
  p.slices = cus * (packed ? 2 : 4);  // of 8 and 4 wavefronts: 16 on a compute unit
  hipStream_t s = static_cast<hipStream_t>(stream);
  const int32_t group = hq / hkv;
  return launched(packed ? launch_shaped_packed(p, group, true, s)
                         : launch_shaped_bf16(p, group, true, s),
                  "attention weights");
}

// Rows of new tokens: the sizes, and where they belong.
neo_status set_rows(PackedRows* p, const void* cache, const int32_t* row_starts, int32_t rows,
                    const int32_t* table, const int32_t* lens, int32_t batch, int32_t mbps,
                    int32_t hkv, int32_t head_dim, int32_t block_size, int32_t num_blocks,
                    int64_t block_stride, bool* noop) {
  *noop = true;
  NEO_TRY(check_sizes(batch, mbps, hkv, head_dim, block_size, num_blocks));
  if (rows < 0) return set_error(NEO_ERR_INVALID_ARG, "rows (%d) is negative", rows);
  if (!row_starts && rows != batch)
    return set_error(NEO_ERR_INVALID_ARG, "without row_starts, rows (%d) must be the batch (%d)",
                     rows, batch);
  if ((int64_t)rows + 15 > (((int64_t)1 << 31) - 1) / hkv)
    return set_error(NEO_ERR_INVALID_ARG, "rows * num_kv_heads must stay below 2^31");
  if (batch == 0 || rows == 0) return ok();
  NEO_TRY(packed_stride(block_stride, hkv, num_blocks, &p->blk_bytes));
  NEO_TRY(check_words(cache, "cache"));
  NEO_TRY(check_ints(row_starts, "row_starts", true));
  NEO_TRY(check_ints(table, "block_table"));
  NEO_TRY(check_ints(lens, "seq_lens"));
  p->cache = static_cast<uint8_t*>(const_cast<void*>(cache));
  p->table = table;
  p->lens = lens;
  p->row_starts = row_starts;
  p->batch = batch;
  p->rows = rows;
  p->mbps = mbps;
  p->hkv = hkv;
  p->num_blocks = num_blocks;
  *noop = false;
  return NEO_OK;
}

neo_status check_row_stride(int64_t stride, const char* name) {
  if (stride < 0 || stride % 8 != 0 || stride > ((int64_t)1 << 30))
    return set_error(NEO_ERR_INVALID_ARG,
                     "%s (%lld) must be a non-negative multiple of 8 elements, at most 2^30", name,
                     (long long)stride);
  return NEO_OK;
}

neo_status evict(void* k, void* v, bool packed, const int32_t* table, const int32_t* lens,
                 const float* sums, int64_t sums_stride, const int32_t* budgets, int32_t recent,
                 const int32_t* new_table, int32_t new_mbps, int32_t* new_lens, int32_t* kept,
                 float* new_sums, int32_t batch, int32_t mbps, int32_t hkv, int32_t head_dim,
                 int32_t block_size, int32_t num_blocks, int64_t stride, void* stream) {
  EvictParams p = {};
  NEO_TRY(check_sizes(batch, mbps, hkv, head_dim, block_size, num_blocks));
  if (recent < 0) return set_error(NEO_ERR_INVALID_ARG, "recent (%d) is negative", recent);
  if (batch == 0) return ok();
  if (new_mbps <= 0)
    return set_error(NEO_ERR_INVALID_ARG, "new_blocks_per_seq (%d) must be positive", new_mbps);
  NEO_TRY(check_sizes(batch, new_mbps, hkv, head_dim, block_size, num_blocks));
  NEO_TRY(packed ? packed_stride(stride, hkv, num_blocks, &p.blk_bytes)
                 : bf16_stride(stride, hkv, num_blocks, &p.blk_bytes));
  NEO_TRY(check_words(k, packed ? "cache" : "k_cache"));
  if (!packed) NEO_TRY(check_words(v, "v_cache"));
  NEO_TRY(check_ints(table, "block_table"));
  NEO_TRY(check_ints(lens, "seq_lens"));
  NEO_TRY(check_ints(sums, "sums"));
  NEO_TRY(check_ints(budgets, "budgets"));
  NEO_TRY(check_ints(new_table, "new_table"));
  NEO_TRY(check_ints(new_lens, "new_lens"));
  NEO_TRY(check_ints(kept, "kept"));
  NEO_TRY(check_ints(new_sums, "new_sums"));
  if (sums_stride < (int64_t)mbps * kBlock)
    return set_error(NEO_ERR_INVALID_ARG,
                     "sums_stride (%lld) must be at least max_blocks_per_seq * block_size",
                     (long long)sums_stride);
  p.k = static_cast<uint8_t*>(k);
  p.v = static_cast<uint8_t*>(v);
  p.table = table;
  p.lens = lens;
  p.sums = sums;
  p.budgets = budgets;
  p.new_table = new_table;
  p.new_lens = new_lens;
  p.kept = kept;
  p.new_sums = new_sums;
  p.sums_stride = sums_stride;
  p.recent = recent;
  p.batch = batch;
  p.hkv = hkv;
  p.mbps = mbps;
  p.new_mbps = new_mbps;
  p.num_blocks = num_blocks;
  return launched(launch_evict(p, packed, static_cast<hipStream_t>(stream)), "eviction");
}

}  // namespace

extern "C" {

neo_status neo_shaped_decode_attention(const void* q, const void* k_cache, const void* v_cache,
                                       const int32_t* block_table, const int32_t* seq_lens,
                                       int32_t num_q_heads, int32_t num_kv_heads,
                                       int32_t head_dim, int32_t block_size, float scale,
                                       const neo_score_shape* shape, float* out, float* lse,
                                       int32_t batch, int32_t max_blocks_per_seq,
                                       int32_t num_blocks, int64_t kv_block_stride,
                                       void* workspace, size_t workspace_bytes, void* stream) {
  return attend(q, {k_cache, v_cache, kv_block_stride}, false, block_table, seq_lens, num_q_heads,
                num_kv_heads, head_dim, block_size, scale, shape, out, lse, batch,
                max_blocks_per_seq, num_blocks, workspace, workspace_bytes, stream);
}

neo_status neo_packed_decode_attention(const void* q, const void* cache,
                                       const int32_t* block_table, const int32_t* seq_lens,
                                       int32_t num_q_heads, int32_t num_kv_heads,
                                       int32_t head_dim, int32_t block_size, float scale,
                                       const neo_score_shape* shape, float* out, float* lse,
                                       int32_t batch, int32_t max_blocks_per_seq,
                                       int32_t num_blocks, int64_t block_stride, void* workspace,
                                       size_t workspace_bytes, void* stream) {
  return attend(q, {cache, nullptr, block_stride}, true, block_table, seq_lens, num_q_heads,
                num_kv_heads, head_dim, block_size, scale, shape, out, lse, batch,
                max_blocks_per_seq, num_blocks, workspace, workspace_bytes, stream);
}

neo_status neo_packed_append(void* cache, const void* k_new, const void* v_new,
                             const int32_t* row_starts, int32_t rows, int64_t k_row_stride,
                             int64_t k_head_stride, int64_t v_row_stride, int64_t v_head_stride,
                             const int32_t* block_table, const int32_t* seq_lens, int32_t batch,
                             int32_t max_blocks_per_seq, int32_t num_kv_heads, int32_t head_dim,
                             int32_t block_size, int32_t num_blocks, int64_t block_stride,
                             void* stream) {
  PackedRows p = {};
  bool noop = false;
  NEO_TRY(check_row_stride(k_row_stride, "k_row_stride"));
  NEO_TRY(check_row_stride(k_head_stride, "k_head_stride"));
  NEO_TRY(check_row_stride(v_row_stride, "v_row_stride"));
  NEO_TRY(check_row_stride(v_head_stride, "v_head_stride"));
  NEO_TRY(set_rows(&p, cache, row_starts, rows, block_table, seq_lens, batch, max_blocks_per_seq,
                   num_kv_heads, head_dim, block_size, num_blocks, block_stride, &noop));
  if (noop) return ok();
  NEO_TRY(check_words(k_new, "k_new"));
  NEO_TRY(check_words(v_new, "v_new"));
  return launched(
      launch_packed_append(p, static_cast<const uint16_t*>(k_new),
                           static_cast<const uint16_t*>(v_new),
                           {k_row_stride, k_head_stride, v_row_stride, v_head_stride},
                           static_cast<hipStream_t>(stream)),
      "packed append");
}

neo_status neo_packed_gather(const void* cache, const int32_t* row_starts, int32_t rows,
                             const int32_t* block_table, const int32_t* seq_lens, int32_t batch,
                             int32_t max_blocks_per_seq, int32_t num_kv_heads, int32_t head_dim,
                             int32_t block_size, int32_t num_blocks, int64_t block_stride,
                             void* k_out, void* v_out, void* stream) {
  PackedRows p = {};
  bool noop = false;
  NEO_TRY(set_rows(&p, cache, row_starts, rows, block_table, seq_lens, batch, max_blocks_per_seq,
                   num_kv_heads, head_dim, block_size, num_blocks, block_stride, &noop));
  if (noop) return ok();
  NEO_TRY(check_words(k_out, "k_out"));
  NEO_TRY(check_words(v_out, "v_out"));
  return launched(launch_packed_gather(p, static_cast<uint16_t*>(k_out),
                                       static_cast<uint16_t*>(v_out),
                                       static_cast<hipStream_t>(stream)),
                  "packed gather");
}

neo_status neo_add_attention_weights(const float* sums, float* sums_out, int64_t sums_stride,
                                     const float* lse, const void* q, const void* k_cache,
                                     const int32_t* block_table, const int32_t* seq_lens,
                                     int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim,
                                     int32_t block_size, float scale,
                                     const neo_score_shape* shape, int32_t batch,
                                     int32_t max_blocks_per_seq, int32_t num_blocks,
                                     int64_t kv_block_stride, void* stream) {
  return add_weights(sums, sums_out, sums_stride, lse, q, {k_cache, nullptr, kv_block_stride},
                     false, block_table, seq_lens, num_q_heads, num_kv_heads, head_dim,
                     block_size, scale, shape, batch, max_blocks_per_seq, num_blocks, stream);
}

neo_status neo_packed_add_attention_weights(const float* sums, float* sums_out,
                                            int64_t sums_stride, const float* lse, const void* q,
                                            const void* cache, const int32_t* block_table,
                                            const int32_t* seq_lens, int32_t num_q_heads,
                                            int32_t num_kv_heads, int32_t head_dim,
                                            int32_t block_size, float scale,
                                            const neo_score_shape* shape, int32_t batch,
                                            int32_t max_blocks_per_seq, int32_t num_blocks,
                                            int64_t block_stride, void* stream) {
  return add_weights(sums, sums_out, sums_stride, lse, q, {cache, nullptr, block_stride}, true,
                     block_table, seq_lens, num_q_heads, num_kv_heads, head_dim, block_size, scale,
                     shape, batch, max_blocks_per_seq, num_blocks, stream);
}

neo_status neo_kv_evict(void* k_cache, void* v_cache, const int32_t* block_table,
                        const int32_t* seq_lens, const float* sums, int64_t sums_stride,
                        const int32_t* budgets, int32_t recent, const int32_t* new_table,
                        int32_t new_blocks_per_seq, int32_t* new_lens, int32_t* kept,
                        float* new_sums, int32_t batch, int32_t max_blocks_per_seq,
                        int32_t num_kv_heads, int32_t head_dim, int32_t block_size,
                        int32_t num_blocks, int64_t kv_block_stride, void* stream) {
  return evict(k_cache, v_cache, false, block_table, seq_lens, sums, sums_stride, budgets, recent,
               new_table, new_blocks_per_seq, new_lens, kept, new_sums, batch, max_blocks_per_seq,
               num_kv_heads, head_dim, block_size, num_blocks, kv_block_stride, stream);
}

neo_status neo_packed_evict(void* cache, const int32_t* block_table, const int32_t* seq_lens,
                            const float* sums, int64_t sums_stride, const int32_t* budgets,
                            int32_t recent, const int32_t* new_table, int32_t new_blocks_per_seq,
                            int32_t* new_lens, int32_t* kept, float* new_sums, int32_t batch,
                            int32_t max_blocks_per_seq, int32_t num_kv_heads, int32_t head_dim,
                            int32_t block_size, int32_t num_blocks, int64_t block_stride,
                            void* stream) {
  return evict(cache, nullptr, true, block_table, seq_lens, sums, sums_stride, budgets, recent,
               new_table, new_blocks_per_seq, new_lens, kept, new_sums, batch, max_blocks_per_seq,
               num_kv_heads, head_dim, block_size, num_blocks, block_stride, stream);
}

}  // extern "C"
