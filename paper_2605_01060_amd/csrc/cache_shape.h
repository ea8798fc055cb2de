// How a call of attention over a cache is cut, from its sizes: the units, who has
// them, and which kernel joins the parts of those that are cut.
#pragma once

#include <stdint.h>

#include <algorithm>

namespace surge {

// Workgroups of a kernel on a CU, by its class (few rows: 16, 32; tiles of 64, 128) and
// d_head, that registers and LDS allow.
constexpr int PLACES[4][3] = {{7, 4, 3}, {5, 3, 2}, {5, 4, 2}, {4, 3, 2}};

// How a call is cut into units: tiles of tile_rows rows (query * group + head
// of the group) of each (sequence, key head).  Their keys, in blocks of
// 1 << block_shift, are shared out to `workers` workgroups, at least least_share blocks
// each, or where that is 0 a unit is a workgroup's.
struct CacheShape {
  int tile_rows, block_shift, least_share;
  bool wave_units;  // a unit is a wave's
  int64_t tiles, units, workers;
  int64_t slot_rows() const { return 2 * workers * tile_rows; }
  int64_t workspace_bytes(int d_head) const {
    return workers ? slot_rows() * (8 + 4 * (int64_t)d_head) + units * 8 : 0;
  }
};

inline CacheShape cache_attention_shape(int64_t n_seqs, int64_t max_rows, int n_kv_heads, int group, int d_head,
                                        int64_t max_length, int n_cus) {
  CacheShape s;
  const int64_t rows = max_rows * group;
  const auto workers_of = [&](int cls) { return (int64_t)n_cus * PLACES[cls][d_head / 64] / 8 * 8; };
  int cls = rows <= 16 ? 0 : rows <= 32 ? 1 : rows <= 64 ? 2 : 3;
  // Against up to 96 keys up to 64 rows, or rows that leave a quarter of their tiles empty,
  // are many waves' units of 32 rows, where those fill the chip: a tile's few blocks don't
  // pay its barriers.  Measured, a tile / waves, us: 841 x 15 x 15, 16 / 4 x 128 43 / 31; 400 x
  // 50 x 64, 16 x 64 32.7 / 27.9; 4000 x about 48 x 48, 12 x 64 257 / 190; 116 x 37 x 37, 32 /
  // 8 x 128 24.5 / 20.8; but 423 x 30 x 30 50 / 55 and 200 x 128 x 128, 12 x 64 23.3 / 26.8.
  const int64_t pieces = (rows + 31) / 32;
  if (cls >= 2 && max_length <= 96 && (cls == 2 || pieces <= 3 * ((rows + 127) / 128)) &&
      n_seqs * n_kv_heads * pieces > workers_of(1))
    cls = 1;
  s.tile_rows = 16 << cls;
  s.block_shift = cls >= 2 ? 6 : 7;  // few rows: 32 keys for each of four waves
  s.tiles = (rows + s.tile_rows - 1) / s.tile_rows;
  s.units = n_seqs * n_kv_heads * s.tiles;
  const int64_t workers = workers_of(cls);
  const int64_t most = ((max_length - 1) >> s.block_shift) + 1;  // blocks of a unit
  // Sharing costs 2 us to find the shares and 5 us for the join, or 13 where tiles'
  // parts are 64 KiB each, a block 1 us (64 keys for a tile, 128 for few rows).  It is
  // left where units are short, or of few rows are more than the chip holds, of tiles
  // more than twice as many.  Measured, a unit a workgroup / shared, us:
  //   30 x 1 x 800, 16 / 4 x 128 10 / 12; 200 x 4 x 500, 12 x 64 23 / 45; 48 x 1 x about
  //   8000, 32 / 8 x 128 111 / 88
  //   (few tiles) 10 x 12 x 1100, 32 / 8 x 128 23 / 18; 1 x 128 x 2000, 8 x 128 47 / 23
  //   (more) 34 x 148 x 1938, 12 x 64 61 / 77; 8 x 2048 x 8192, 16 x 128 1047 / 1144
  s.least_share = cls >= 2 ? 8 : 2;
  s.workers = 0;
  if (most > (cls >= 2 ? (s.units <= workers / 4 ? 16 : 32) : 8) && n_seqs * s.tiles <= 2048 && s.units * most < (1 << 30) &&
      s.units <= (cls >= 2 ? 2 : 1) * workers)
    s.workers = workers;
  // Where units of few rows are short, or very many and not long, a wave has one for
  // itself: no waves without keys and no join of four.  Measured, a workgroup / a wave, us:
  // 400 x 1 x 60, 32 / 8 x 128 17.0 / 11.2; 200 x 8 x 100, 16 / 4 x 128 15.0 / 10.5; 1000 x 8 x
  // 240, 32 / 8 x 128 113 / 89, 1000 x 8 x 1024 286 / 254, 800 x 1 x 1024 162 / 173; but 140 x 1
  // x 240 12.2 / 14.0 and 400 x 1 x 900 80 / 92.  max_length says nothing of most sequences,
  // but one may be as long, and the call then waits for its wave: among 800 x 1 of about 200
  // keys, 32 / 8 x 128, one of 1024 43 / 40, of 2048 43 / 66, of 30,000 212 / 773.
  s.wave_units = cls < 2 && s.workers == 0 && s.units > workers &&
                 (max_length <= 128 || (max_length <= 1024 && s.units >= 8 * workers));
  return s;
}

// Waves that join the parts of a row, or 0: of eight rows, in turn.  By the parts that a
// unit is cut into, about: its rows' join has as many waves as they keep busy (by the
// workers alone 4 x 128 x 1500, 12 x 64 took 40 us, not 19).
inline int cache_attention_join(const CacheShape& s, int64_t max_length) {
  const int64_t blocks = ((max_length - 1) >> s.block_shift) + 1;
  const int64_t parts = std::min(s.workers / s.units, blocks / s.least_share);
  return parts >= 16 ? 16 : parts >= 4 ? 4 : s.tile_rows < 64 ? 1 : 0;
}

}  // namespace surge
