// Cross attention's work list.
#include <algorithm>
#include <functional>
#include <queue>

#include "cross_list.h"

namespace surge {
namespace {

int64_t blocks32(int64_t n) { return (n + 31) / 32; }

struct Lengths {
  int64_t n_seqs;
  const int64_t *cu_q, *cu_kv;
  int group;
  int64_t rows(int64_t i) const { return (cu_q[i + 1] - cu_q[i]) * group; }
  int64_t keys(int64_t i) const { return cu_kv[i + 1] - cu_kv[i]; }
};

// Units of at most `share` 32-key blocks: a sequence with more is split into
// equal parts.
CrossList split_list(const Lengths& s, int64_t share) {
  CrossList out;
  for (int64_t i = 0; i < s.n_seqs; ++i) {
    const int64_t rows = s.rows(i), keys = s.keys(i), kb = blocks32(keys);
    const int64_t parts = kb > share ? (kb + share - 1) / share : 1;
    const int64_t per = (kb + parts - 1) / parts * 32;  // keys of a part
    // The class of the fewest rows that holds them.
    const int cls = rows > 64 ? 0 : rows > 32 ? 1 : 2;
    const int64_t step = CROSS_ROWS[cls];
    std::vector<CrossItem>& items = out.items[cls];
    for (int64_t r = 0; r < rows; r += step) {
      CrossItem it = {(int32_t)s.cu_q[i], (int32_t)r, (int32_t)rows, (int32_t)s.cu_kv[i], 0,
                      (int32_t)keys, -1, 0};
      if (parts == 1) {
        items.push_back(it);
        continue;
      }
      const int32_t blocks = (int32_t)blocks32(std::min(step, rows - r));
      const int32_t part0 = (int32_t)out.n_parts;
      int32_t n = 0;
      for (int64_t k = 0; k < keys; k += per, ++n) {
        it.k0 = (int32_t)k;
        it.k1 = (int32_t)std::min(keys, k + per);
        it.part = part0 + n * blocks;
        items.push_back(it);
      }
      out.n_parts += (int64_t)n * blocks;
      out.max_parts = std::max(out.max_parts, (int)n);
      for (int32_t b = 0; b < blocks; ++b)
        out.joins.push_back({(int32_t)s.cu_q[i], (int32_t)r + 32 * b,
                             (int32_t)std::min<int64_t>(32, rows - r - 32 * b), part0 + b, n, blocks});
    }
  }
  for (std::vector<CrossItem>& items : out.items)
    std::stable_sort(items.begin(), items.end(), [](const CrossItem& a, const CrossItem& b) {
      return a.k1 - a.k0 > b.k1 - b.k0;
    });
  return out;
}

// What a list takes, in us: each class as its units, longest first, go to the
// first free of the chip's places, then the join.  A place is a workgroup that
// the registers let a CU hold (of one wave the four that keep the memory
// busy).  Measured on full chips, a block of 32 keys takes 128 rows 0.67, 0.92
// and 1.10 us (d_head 32, 64, 128), and a unit about six blocks beside its
// keys.
double list_us(const CrossList& list, int n_kv_heads, int d_head, int n_cus) {
  const double block = d_head == 32 ? 0.67 : d_head == 64 ? 0.92 : 1.10;
  const int per_cu[CROSS_CLASSES] = {d_head == 128 ? 2 : 3, 4, 4};
  double us = 0;
  for (int c = 0; c < CROSS_CLASSES; ++c) {
    std::priority_queue<double, std::vector<double>, std::greater<double>> places;
    double end = 0;
    for (const CrossItem& it : list.items[c])
      for (int h = 0; h < n_kv_heads; ++h) {
        double t = (double)(blocks32(it.k1 - it.k0) + 6) * block;
        if ((int)places.size() == per_cu[c] * n_cus) {
          t += places.top();
          places.pop();
        }
        places.push(t);
        end = std::max(end, t);
      }
    us += end;
  }
  if (list.n_parts > 0) us += 5 + (double)list.n_parts * n_kv_heads * 32 * (d_head * 8 + 16) / 4e6;
  return us;
}

}  // namespace

// No unit has more than its share of the key blocks, a share being what one
// of 4 to 8 waves per CU would have of all of them, and at least 8 (256
// keys).  Few large units leave CUs idle at the end, many cost the join, and
// which is less depends on the lengths: where the units are few the list with
// the least time by list_us is taken.  Measured (us, 4 / 6 / 8 waves per CU): heads
// 16 / 4 x 128, four texts of about 6000, 1500 queries each, 313 / 343 / 345;
// 16 x 64, 7 texts of about 5000, 300 queries, 160 / 162 / 136; 12 x 64, two
// of about 9000, 2000 queries, 121 / 91 / 111; 12 x 32, one of 4000, 500
// queries, 20.8 / 17.8 / 23.1.  One wave's units are bound by the stream of
// the keys, which 4 per CU keep up best: 16 x 64, three texts of about 20,000,
// one query, 47.7 / 52.8 / 53.0.
void build_cross_list(int64_t n_seqs, const int64_t* cu_q, const int64_t* cu_kv, int n_kv_heads,
                      int group, int d_head, int n_cus, CrossList* out) {
  const Lengths s = {n_seqs, cu_q, cu_kv, group};
  int64_t work = 0, longest = 0;
  bool wide = false;
  for (int64_t i = 0; i < n_seqs; ++i) {
    const int64_t rows = s.rows(i), kb = blocks32(s.keys(i));
    work += blocks32(rows) * kb * n_kv_heads;
    if (rows > 0) longest = std::max(longest, kb);
    wide = wide || rows > 32;
  }
  auto share = [&](int per_cu) {
    const int64_t waves = (int64_t)n_cus * per_cu;
    return std::max<int64_t>(8, (work + waves - 1) / waves);
  };
  *out = split_list(s, share(4));
  size_t units = 0;
  for (const auto& items : out->items) units += items.size() * n_kv_heads;
  if (!wide || longest <= share(8) || units > (size_t)n_cus * 8) return;
  double best = list_us(*out, n_kv_heads, d_head, n_cus);
  for (int per_cu : {6, 8}) {
    CrossList list = split_list(s, share(per_cu));
    const double us = list_us(list, n_kv_heads, d_head, n_cus);
    if (us < best) {
      best = us;
      *out = std::move(list);
    }
  }
}

}  // namespace surge
