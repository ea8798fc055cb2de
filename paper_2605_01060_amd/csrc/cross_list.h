// Cross attention's work list, built on the host from the lengths.
#pragma once

#include <stdint.h>

#include <vector>

namespace surge {

// Units of work by the rows that they hold.
constexpr int CROSS_CLASSES = 3;
constexpr int CROSS_ROWS[CROSS_CLASSES] = {128, 64, 32};

// Up to CROSS_ROWS[class] rows of one sequence over keys k0 .. k1 - 1 of its
// text.
struct CrossItem {
  int32_t q_beg;   // first query token of the sequence
  int32_t row0;    // first row (query * group + head of the group)
  int32_t rows;    // rows of the sequence
  int32_t kv_beg;  // first key row of its text
  int32_t k0, k1;
  int32_t part;    // slot of its first 32 rows' partial result, the others'
                   // behind it; -1: the unit has all keys
  int32_t reserved;
};

// 32 rows whose keys are split over slots part0, part0 + stride, ...
struct CrossJoin {
  int32_t q_beg, row0, rows;  // rows: of these 32, how many there are
  int32_t part0, parts, stride;
};

struct CrossList {
  std::vector<CrossItem> items[CROSS_CLASSES];  // longest first
  std::vector<CrossJoin> joins;
  int64_t n_parts = 0;                  // slots
  int max_parts = 0;                    // of one join
  bool short_blocks = false;            // 128 rows against 32 keys, not 64
};
// cu_q, cu_kv: checked.  n_cus: compute units to fill.
void build_cross_list(int64_t n_seqs, const int64_t* cu_q, const int64_t* cu_kv, int n_kv_heads,
                      int group, int d_head, int n_cus, CrossList* out);

}  // namespace surge
