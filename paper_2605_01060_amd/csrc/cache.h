// Launchers of the operators of a decoder: its keys and values in 4 bits,
// attention over them, and the check of drafted tokens.  The caller has
// checked the arguments.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "cache_shape.h"

namespace surge {

// Pages of tokens, see surge_kv_cache.  A page holds for every key head, in
// turn: the codes of its keys [tokens, d_head / 2 bytes], of its values, the
// scales of its keys [tokens, d_head / 32 bytes], of its values.
struct CacheView {
  uint8_t* pages;
  int64_t n_pages, page_bytes;
  int page_shift, n_kv_heads, n_seqs, max_length;
  const int32_t* table;
  int64_t ld_table;
  const int32_t* lengths;
};

// The rows of a call: sequence i has rows cu[i] .. cu[i+1]-1, or `each` rows
// where cu is NULL, of n_rows in all.  They are its last positions.
struct CacheRows {
  const int32_t* cu;
  int n_rows, each;
};

struct CacheStore {
  CacheView c;
  CacheRows r;
  uint16_t *k, *v;  // read by a write, written by a read
  int64_t ld_k, ld_v;
  int heads_each;  // of a wave: the launch's
};
int64_t cache_store_blocks(int64_t n_rows, int n_kv_heads, int d_head);  // of 256 threads, of a launch
hipError_t launch_cache_write(CacheStore a, int d_head, hipStream_t stream);
hipError_t launch_cache_read(CacheStore a, int d_head, hipStream_t stream);

// What a kernel divides a number below 2^31 by d with.
struct Divisor {
  uint32_t m;
  int s;
};
Divisor divisor(int d);  // d >= 1

struct CacheAttention {
  CacheView c;
  CacheRows r;
  const uint16_t* q;
  uint16_t* out;
  int64_t ld_q, ld_out;
  int group, max_rows;
  bool causal;
  float scale_log2;   // scale * log2(e)
  // Of cache_attention_shape, and of cache_attention_join.
  int tile_rows, block_shift, tiles, units, workers, least_share, join_waves;
  bool wave_units;
  Divisor by_group, by_tiles, by_heads, by_units, by_workers;  // by_units: by n_seqs * n_kv_heads
  // Workspace, where there are workers: of the two slots that each has for the
  // parts of its first and last unit, the rows' maxima (in log2 units) and sums,
  // their outputs, and which workers have the parts of a unit.
  float* part_o;     // [slot, row, d_head]
  float2* part_ml;   // [slot, row]
  int2* joins;       // [unit] first and last worker; first < 0: not cut
};

hipError_t launch_cache_attention(const CacheAttention& a, int d_head, hipStream_t stream);

struct VerifyDrafts {
  int max_drafts, vocab;
  const int32_t *n_drafts, *drafts;  // n_drafts NULL: max_drafts each
  const float *p, *q;                // q NULL: drafts of probability 1
  int64_t ld_p, ld_q;
  const float* u;
  int32_t *tokens, *accepted;
  double* sums;  // workspace of verify_workspace bytes
};
int64_t verify_workspace(int64_t n_seqs, int vocab);
hipError_t launch_verify_drafts(int64_t n_seqs, const VerifyDrafts& a, hipStream_t stream);

}  // namespace surge
