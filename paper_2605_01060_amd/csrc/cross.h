// Cross attention's launcher.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "cross_list.h"

namespace surge {

struct CrossAttention {
  const uint16_t *q, *k, *v;
  int64_t ld_q, ld_k, ld_v;
  const uint8_t* mask;  // [keys], 0 = left out; NULL: none
  float scale_log2;     // scale * log2(e)
  int n_kv_heads, group;
  const CrossItem* items;         // class by class
  int n_items[CROSS_CLASSES];
  const CrossJoin* joins;
  int n_joins, max_parts;
  bool short_blocks;  // 128 rows of 128-dimensional heads against 32 keys
  float2* part_ml;  // [part, key head, 32] (maximum in log2 units, sum)
  float* part_o;    // [part, key head, 32, d_head]
  uint16_t* out;
  int64_t ld_out;
};
hipError_t launch_cross_attention(const CrossAttention& a, int d_head, hipStream_t stream);

}  // namespace surge
