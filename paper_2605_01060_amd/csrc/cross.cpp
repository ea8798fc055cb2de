// Cross attention's work list.
#include <algorithm>

#include "cross_list.h"

namespace surge {

void build_cross_list(int64_t n_seqs, const int64_t* cu_q, const int64_t* cu_kv, int n_kv_heads,
                      int group, int n_cus, CrossList* out) {
  // Keys are split so that no unit has more than its share of the key blocks
  // of a chip of eight waves per CU, and at least eight blocks of 32.
  auto row_blocks = [&](int64_t i) { return ((cu_q[i + 1] - cu_q[i]) * group + 31) / 32; };
  auto key_blocks = [&](int64_t i) { return (cu_kv[i + 1] - cu_kv[i] + 31) / 32; };
  int64_t work = 0;
  for (int64_t i = 0; i < n_seqs; ++i) work += row_blocks(i) * key_blocks(i) * n_kv_heads;
  const int64_t waves = (int64_t)n_cus * 8;
  const int64_t share = std::max<int64_t>(8, (work + waves - 1) / waves);
  for (int64_t i = 0; i < n_seqs; ++i) {
    const int64_t rows = (cu_q[i + 1] - cu_q[i]) * group, keys = cu_kv[i + 1] - cu_kv[i];
    const int64_t kb = key_blocks(i);
    const int64_t parts = kb > share ? (kb + share - 1) / share : 1;
    const int64_t per = (kb + parts - 1) / parts * 32;  // keys of a part
    for (int64_t r = 0; r < rows; r += 32) {
      CrossItem it = {(int32_t)cu_q[i], (int32_t)r, (int32_t)rows, (int32_t)cu_kv[i], 0, (int32_t)keys,
                      -1,               0};
      if (parts == 1) {
        out->items.push_back(it);
        continue;
      }
      CrossJoin j = {(int32_t)cu_q[i], (int32_t)r, (int32_t)std::min<int64_t>(32, rows - r),
                     (int32_t)out->n_parts, 0};
      for (int64_t k = 0; k < keys; k += per) {
        it.k0 = (int32_t)k;
        it.k1 = (int32_t)std::min(keys, k + per);
        it.part = (int32_t)out->n_parts++;
        ++j.parts;
        out->items.push_back(it);
      }
      out->joins.push_back(j);
    }
  }
  std::stable_sort(out->items.begin(), out->items.end(), [](const CrossItem& a, const CrossItem& b) {
    return a.k1 - a.k0 > b.k1 - b.k0;
  });
}

}  // namespace surge
