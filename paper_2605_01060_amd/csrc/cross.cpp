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

// Units of at most `share` (>= 1) 32-key blocks: a sequence with more is split
// into equal parts.
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

// What a unit of a class takes, measured (us): `chain` for a block of 32 keys
// where it is alone, `full` where the chip is full of such units, `places` of
// them on a CU (registers and LDS), and `base` beside its keys.  The units of
// one or two waves are bound by the stream of their keys where they are many.
struct UnitCost {
  int places;
  double base, chain, full;
};
UnitCost unit_cost(int cls, int d_head, bool short_blocks) {
  static const UnitCost costs[CROSS_CLASSES][3] = {
      {{5, 2.9, 0.31, 0.98}, {4, 3.2, 0.47, 1.13}, {2, 4.3, 0.60, 1.03}},
      {{14, 2.6, 0.47, 0.47}, {8, 3.0, 0.58, 0.58}, {4, 3.7, 0.80, 0.80}},
      {{19, 2.4, 0.46, 0.46}, {9, 2.5, 0.62, 0.62}, {4, 2.9, 0.94, 0.94}},
  };
  if (short_blocks) return {3, 4.0, 0.80, 1.47};
  return costs[cls][d_head / 64];
}

// What the units of a class take, in us: longest first they go to the first
// free of the chip's places, or their keys come from memory.
double class_us(const CrossList& list, int cls, int n_kv_heads, int d_head, bool short_blocks, int n_cus) {
  const int64_t units = (int64_t)list.items[cls].size() * n_kv_heads;
  if (units == 0) return 0;
  const UnitCost q = unit_cost(cls, d_head, short_blocks);
  const double load = std::min(1.0, (double)units / ((double)n_cus * q.places));
  const double block = std::max(q.chain, q.full * load);
  std::priority_queue<double, std::vector<double>, std::greater<double>> places;
  double end = 0, keys = 0;
  for (const CrossItem& it : list.items[cls]) {
    keys += it.k1 - it.k0;
    for (int h = 0; h < n_kv_heads; ++h) {
      double t = q.base + (double)blocks32(it.k1 - it.k0) * block;
      if ((int)places.size() == q.places * n_cus) {
        t += places.top();
        places.pop();
      }
      places.push(t);
      end = std::max(end, t);
    }
  }
  if (cls > 0) end = std::max(end, q.base + keys * n_kv_heads * d_head * 4 / 4.9e6);
  return end;
}

// What a list takes, with the better of the two blocks for units of 128 rows
// of 128-dimensional heads, and the join, which reads its parts at 5.7 TB/s
// (measured where they have just been written: 68 MB in 14 us).
double list_us(CrossList* list, int n_kv_heads, int d_head, int n_cus) {
  double us = class_us(*list, 0, n_kv_heads, d_head, false, n_cus);
  list->short_blocks = false;
  if (d_head == 128) {
    const double other = class_us(*list, 0, n_kv_heads, d_head, true, n_cus);
    list->short_blocks = other < us;
    us = std::min(us, other);
  }
  for (int c = 1; c < CROSS_CLASSES; ++c) us += class_us(*list, c, n_kv_heads, d_head, false, n_cus);
  if (list->n_parts > 0)
    us += 2.7 + (double)list->n_parts * n_kv_heads * 32 * (d_head * 8 + 16) / 5.7e6;
  return us;
}

}  // namespace

// A unit has at most its share of the key blocks, a share being what one of 4
// to 8 waves per CU would have of all of them, and at least two, or all keys
// of its rows.  Few large units leave CUs idle at the end or wait for one
// wave's chain of blocks, many cost the join, and which is less depends on the
// lengths: the list with the least time by list_us is taken.  Measured (us,
// whole, then shares of 4 / 6 / 8 waves per CU, * the list taken):
//   texts x queries x keys, heads
//   4 x 1500 x about 6000, 16 / 4 x 128   317, 316 / 314 / 284*
//   3 x 1500 x 15,000, 8 / 1 x 128        379, 381 / 330 / 330*
//   6 x 500 x 10,000, 16 / 4 x 128        275*, 275 / 260 / 260
//   7 x 300 x 5000, 16 x 64               98, 98 / 83 / 83*
//   2 x 2000 x 9000, 12 x 64              174, 175 / 153 / 153*
//   10 x 300 x 2000, 8 x 128              43.7*, 49.4 / 49.4 / 49.2
//   1 x 1000 x 1000, 16 / 4 x 128         24.0, 25.9* / 28.5 / 28.3
//   1 x 256 x 50,000, 8 x 128             946, 88 / 88 / 81*
//   2 x 100 x 30,000, 12 x 32             333, 52 / 43 / 41*
//   3 x 40 x 20,000, 16 x 64              385, 63* / 50 / 48
//   3 x 1 x about 20,000, 16 x 64         517, 38* / 41 / 42
//   64 x 1 x about 96, 16 x 64            7.2*, 9.0 / 9.2 / 10.0
//   1 x 1 x 512, 12 x 64                  12.7, 6.9* / 6.8 / 6.8
// The list taken is 3 % behind the best of these on the mean, 28 % in the call of
// 40 queries.
void build_cross_list(int64_t n_seqs, const int64_t* cu_q, const int64_t* cu_kv, int n_kv_heads,
                      int group, int d_head, int n_cus, CrossList* out) {
  const Lengths s = {n_seqs, cu_q, cu_kv, group};
  // longest: key blocks of the longest text that is read, a share of them where
  // none is split.  Texts without queries do not count, so it may be that only
  // they have states: one block then, as a share of none has no parts.
  int64_t work = 0, longest = 1, units = 0;
  for (int64_t i = 0; i < n_seqs; ++i) {
    const int64_t rows = s.rows(i), kb = blocks32(s.keys(i));
    work += blocks32(rows) * kb * n_kv_heads;
    units += (rows > 64 ? (rows + 127) / 128 : rows > 0) * n_kv_heads;
    if (rows > 0) longest = std::max(longest, kb);
  }
  auto share = [&](int per_cu) {
    const int64_t waves = (int64_t)n_cus * per_cu;
    return std::max<int64_t>(2, (work + waves - 1) / waves);
  };
  // Of many units only the longest matter: they are split where one alone
  // would take a good part of the whole.  Blocks of 32 and of 64 keys are within
  // 1 % of each other there but for the shortest texts (500 sequences, 128
  // queries, 192 / 288 keys, 8 heads x 128: 64 keys 124 / 165, 32 keys 125 / 163
  // us) and for lengths that differ (60, 300, about 1500: 166 / 161).
  if (units > 8 * (int64_t)n_cus) {
    *out = split_list(s, longest > share(4) ? std::max<int64_t>(16, share(4)) : longest);
    out->short_blocks = d_head == 128 && longest > 8;
    return;
  }
  *out = split_list(s, longest);
  double best = list_us(out, n_kv_heads, d_head, n_cus);
  int64_t last = longest;
  for (int per_cu : {4, 6, 8}) {
    if (share(per_cu) >= last) continue;
    last = share(per_cu);
    CrossList list = split_list(s, last);
    const double us = list_us(&list, n_kv_heads, d_head, n_cus);
    if (us < best) {
      best = us;
      *out = std::move(list);
    }
  }
}

}  // namespace surge
