// Cross attention's work list, built on the host from the lengths.
#pragma once

#include <stdint.h>

#include <vector>

namespace surge {

// 32 rows of one sequence over keys k0 .. k1 - 1 of its text.
struct CrossItem {
  int32_t q_beg;   // first query token of the sequence
  int32_t row0;    // first row (query * group + head of the group)
  int32_t rows;    // rows of the sequence
  int32_t kv_beg;  // first key row of its text
  int32_t k0, k1;
  int32_t part;    // slot of the partial result, -1: the unit has all keys
  int32_t reserved;
};

// 32 rows whose keys are split over parts part0 .. part0 + parts - 1.
struct CrossJoin {
  int32_t q_beg, row0, rows;  // rows: of these 32, how many there are
  int32_t part0, parts;
};

struct CrossList {
  std::vector<CrossItem> items;  // longest first
  std::vector<CrossJoin> joins;
  int64_t n_parts = 0;
};
// cu_q, cu_kv: checked.  n_cus: compute units to fill.
void build_cross_list(int64_t n_seqs, const int64_t* cu_q, const int64_t* cu_kv, int n_kv_heads,
                      int group, int n_cus, CrossList* out);

}  // namespace surge
