// Launchers of attention with shaped scores, of the packed cache's operations and
// of eviction.
#pragma once

#include "neo_internal.h"

namespace neo {

struct ShapedParams;
// weights: the sums of the weights instead of attention.
hipError_t launch_shaped_bf16(const ShapedParams& p, int32_t group, bool weights,
                              hipStream_t stream);
hipError_t launch_shaped_packed(const ShapedParams& p, int32_t group, bool weights,
                                hipStream_t stream);

// Rows of new tokens and where they belong: request b's are row_starts[b] ..
// row_starts[b + 1] - 1 (null: row b), its last tokens.
struct PackedRows {
  uint8_t* cache;
  int64_t blk_bytes;
  const int32_t* table;
  const int32_t* lens;
  const int32_t* row_starts;
  int32_t batch, rows, mbps, hkv, num_blocks;
};
// Row and head strides in elements.
struct RowStrides {
  int64_t k_row, k_head, v_row, v_head;
};
hipError_t launch_packed_append(const PackedRows& p, const uint16_t* k_new, const uint16_t* v_new,
                                const RowStrides& s, hipStream_t stream);
hipError_t launch_packed_gather(const PackedRows& p, uint16_t* k_out, uint16_t* v_out,
                                hipStream_t stream);

struct EvictParams {
  uint8_t* k;               // K of the bf16 cache, or the packed cache
  uint8_t* v;               // V of the bf16 cache
  int64_t blk_bytes;
  const int32_t* table;     // [batch][mbps]
  const int32_t* lens;
  const float* sums;        // [batch][hkv][sums_stride]
  const int32_t* budgets;   // [batch]
  const int32_t* new_table; // [batch][new_mbps]
  int32_t* new_lens;        // [batch]
  int32_t* kept;            // [batch][hkv][16 * new_mbps]
  float* new_sums;          // [batch][hkv][16 * new_mbps]
  int64_t sums_stride;
  int32_t recent;
  int32_t batch, hkv, mbps, new_mbps, num_blocks;
};
hipError_t launch_evict(const EvictParams& p, bool packed, hipStream_t stream);

}  // namespace neo
