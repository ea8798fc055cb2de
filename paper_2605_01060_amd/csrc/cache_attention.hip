// Attention over a cache in 4 bits (gfx950, bf16 MFMA, fp32 softmax).
//
//   out[t, h] = sum_k p_k V[k, h / G] / sum_k p_k,
//   p_k = exp(scale Q[t, h] . K[k, h / G]) over the positions that row t sees,
//
// G = heads per key head; a row that sees none gives zeros.  The G query heads
// that share a key head are rows of one matrix: row r of (sequence, key head) is
// query r / G, head r % G of the group.
//
// A code is decoded to bf16 exactly, two by one instruction that takes the scale's
// exponent, so what is rounded is what cross attention rounds: the probabilities to
// bf16 for their product with V, not in their sum.  S^T = K Q^T and O^T += V^T P^T,
// so that a lane owns a row's maximum, sum and rescaling and the probabilities are
// the second product's operand where they are.  Three arrangements, by the rows of a
// (sequence, key head) in the call (and see cache_attention_shape):
//
// Up to 16 or 32 rows (a step, drafts): waves with blocks of 32 keys of their own
// against all rows in 16x16x32 MFMAs.  A lane loads a quarter of a key, whose codes
// are the MFMA's operand as they come (the order of the features is one for both
// operands), so K needs no LDS; V goes through it to be read transposed.  The next
// block's codes are loaded while one is computed (two ahead changed nothing).  Bound
// by memory where there is much of it: one query of 32 / 8 heads x 128 over 48 x about
// 8,000 keys takes 84 us, 5.2 TB/s, over 100,003 keys 25 us, of which the first 4 find
// the share and the first codes.  The VALU is half busy then, a half of it decoding.
//
// 64 or 128 rows a tile (prompts, many drafts): four waves decode blocks of 64 keys
// into LDS together, a block ahead, and take 32x32x16 MFMAs from there; for 64 rows
// two waves share 32 rows and halve the keys (64 x 16 queries x 3001 keys, 16 / 4 x
// 128: 97 -> 61 us against waves with keys of their own).  8 x 2048 queries x 8192
// keys, 16 x 128: 1,059 us, 1,039 TFLOP/s, 16 x 64 620 us, 886 TFLOP/s, 16 x 32 476
// us; what bounds it is the power limit and the VALU, as in cross attention.  Blocks
// of 32 keys with three units a CU were 4 to 11 % slower here.
//
// Lengths are known on the device alone.  Where a unit (a tile of a sequence and key
// head) has a long way to go and units are few, all units' blocks of keys are shared
// out evenly to as many workgroups as the chip holds, each of which finds its share
// from the lengths (2 to 3 us); a second kernel joins the parts of a unit that is cut.
// 4 x about 1500 queries x about 6000 keys, 16 / 4 x 128: 384 us with a unit a
// workgroup, 252 so.  Otherwise a unit is a workgroup's, or where it is short a wave's,
// the last tiles of all sequences first; sequences are in their order, whatever their
// lengths, so that one long one among many is waited for (cache_shape.h).
#include <float.h>
#include <math.h>

#include <algorithm>

#include "cache_device.h"

namespace surge {
namespace {

// The 16 bytes of codes (d_head 128; 8 or 4 for smaller heads) of a quarter of
// a key or value.
template <int DH>
struct Quarter {
  static constexpr int DWORDS = DH / 32;
  uint32_t w[DWORDS];
  __device__ __forceinline__ void load(const uint8_t* p) {
    if constexpr (DWORDS == 4) {
      const u32x4 v = *reinterpret_cast<const u32x4*>(p);
      w[0] = v[0], w[1] = v[1], w[2] = v[2], w[3] = v[3];
    } else if constexpr (DWORDS == 2) {
      const uint2 v = *reinterpret_cast<const uint2*>(p);
      w[0] = v.x, w[1] = v.y;
    } else {
      w[0] = *reinterpret_cast<const uint32_t*>(p);
    }
  }
};

// x / d for x < 2^31: m = ceil(2^(31 + s) / d) with 2^s >= d is off from 2^(31 + s) /
// d by less than 2^-31 of it.
__device__ __forceinline__ int over(int x, const Divisor& d) {
  return (int)(__umulhi((uint32_t)x << 1, d.m) >> d.s);
}

// A sequence's rows: the first one's number and position, how many there are
// (queries * group), and the sequence's length.
struct Sequence {
  int q_beg, rows, first, length;
};

__device__ __forceinline__ Sequence sequence_of(const CacheAttention& a, int seq) {
  Sequence s;
  int n;
  if (a.r.cu) {
    s.q_beg = min(max(a.r.cu[seq], 0), a.r.n_rows);
    n = min(max(a.r.cu[seq + 1], s.q_beg), a.r.n_rows) - s.q_beg;
  } else {
    s.q_beg = seq * a.r.each;
    n = a.r.each;
  }
  s.length = length_of(a.c, seq);
  s.first = s.length - n;
  s.rows = min(n, a.max_rows) * a.group;
  return s;
}

// A value that all lanes of a wave have, in a scalar register.
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ Sequence uniform(const Sequence& s) {
  return {uniform(s.q_beg), uniform(s.rows), uniform(s.first), uniform(s.length)};
}

// The lane's number, made anew where it is asked for: what a unit's code makes of it
// is not kept in registers from unit to unit (up to 50 of them).
__device__ __forceinline__ int own_lane() {
  int lane = threadIdx.x & 63;
  asm volatile("" : "+v"(lane));
  return lane;
}

// A unit of work: a tile of rows of one (sequence, key head), with all of the keys
// that they see or a part of them.
struct Unit {
  int seq, kvh, row0;         // row0: first row of the tile, in the sequence
  int q_beg, rows, first;     // of the sequence
  int limit;                  // keys that the tile's last row sees
  int k0, k1;                 // keys of the unit
  bool whole;                 // these are all of its rows' keys
  int slot;                   // of its part, where not
};

// Keys that a row sees.
__device__ __forceinline__ int row_limit(const CacheAttention& a, const Unit& u, int row) {
  return a.causal ? u.first + over(row, a.by_group) + 1 : u.limit;
}

// Keys that the last row of tile `tile` sees; blocks of them, one at least, 0 for
// a tile without rows.
__device__ __forceinline__ int limit_of(const CacheAttention& a, const Sequence& s, int tile) {
  const int last = min((tile + 1) * a.tile_rows, s.rows) - 1;
  return a.causal ? max(s.first + over(last, a.by_group) + 1, 0) : s.length;
}
__device__ __forceinline__ int blocks_of(const CacheAttention& a, const Sequence& s, int tile) {
  if (tile * a.tile_rows >= s.rows) return 0;
  return max((limit_of(a, s, tile) + (1 << a.block_shift) - 1) >> a.block_shift, 1);
}

// With all of its keys.
__device__ __forceinline__ Unit unit_of(const CacheAttention& a, const Sequence& s, int seq, int kvh, int tile) {
  Unit u;
  u.seq = seq;
  u.kvh = kvh;
  u.row0 = tile * a.tile_rows;
  u.q_beg = s.q_beg;
  u.rows = s.rows;
  u.first = s.first;
  u.limit = limit_of(a, s, tile);
  u.k0 = 0;
  u.k1 = u.limit;
  u.whole = true;
  u.slot = 0;
  return u;
}

__device__ __forceinline__ int scan64(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, true);  // of lanes 1, 2, 4, 8 before in a row
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, true);  // of the last lane of the row, the half before
  return v + __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, true);
}

// A unit a workgroup (or wave), the last tiles first, whose rows see the most keys.
template <class Body>
__device__ __forceinline__ void one_unit(const CacheAttention& a, int index, Body body) {
  const int of_tile = over(index, a.by_units);
  const int rest = index - of_tile * (a.c.n_seqs * a.c.n_kv_heads), tile = a.tiles - 1 - of_tile;
  const int seq = over(rest, a.by_heads);
  const Sequence s = uniform(sequence_of(a, seq));
  if (tile * a.tile_rows < s.rows) body(unit_of(a, s, seq, rest - seq * a.c.n_kv_heads, tile));
}

// Sums of a value over the workgroup's threads before this one, and over all.
__device__ __forceinline__ int2 sums_before(int v, int* s_wave) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int upto = scan64(v);
  if (lane == 63) s_wave[wave] = upto;
  __syncthreads();
  int before = upto - v, total = 0;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    if (w < wave) before += s_wave[w];
    total += s_wave[w];
  }
  return make_int2(before, uniform(total));
}

// The last of 256 increasing numbers that is at most `at`.
__device__ __forceinline__ int last_upto(const int* before, int at) {
  int n = -1;
#pragma unroll
  for (int i = 0; i < 4; ++i) n += __popcll(__ballot(before[i * 64 + (threadIdx.x & 63)] <= at));
  return uniform(n);
}

// The largest of the workgroup's values, none below 0.
__device__ __forceinline__ int most_of(int v, int* s_wave) {
  v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, true));  // as scan64
  v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, true));
  v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, true));
  v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, true));
  v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, true));
  v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, true));
  if ((threadIdx.x & 63) == 63) s_wave[threadIdx.x >> 6] = v;
  __syncthreads();
  return uniform(max(max(s_wave[0], s_wave[1]), max(s_wave[2], s_wave[3])));
}

// The workgroup's number among `active` ones, -1 without one: those of one XCD
// follow each other, and every XCD has as many.
__device__ __forceinline__ int worker_of(int active) {
  const int each = (active + 7) >> 3, mine = (int)blockIdx.x >> 3;
  const int worker = ((int)blockIdx.x & 7) * each + mine;
  return mine < each && worker < active ? worker : -1;
}

// The workgroup's part of all units' blocks of keys.  Workgroups of one XCD have
// parts next to each other, of a sequence's keys, in the order of sequence, tile,
// key head; every XCD has as many.
//
// Few units are cut into equal parts, the most that the workers suffice for, so that
// no worker has two: a unit's start and end take 5 us.  Of more units each worker has
// an equal share, which starts and ends anywhere, or, where they are no more than the
// workers and the longest is within what a cut would save (`fit`), a whole unit.  The
// parts of a unit that is cut are joined afterwards; who has the last one knows where
// they started.  Measured, us, a unit a workgroup / equal shares / equal parts:
//   16 x 5 queries x about 3001 keys, 16 / 4 x 128    41 / 22 / 20
//   64 x 5 x about 3001, 16 / 4 x 128                 42 / 39 / 46
//   48 x 1 x about 8000, 32 / 8 x 128                 111 / 88 / 106
//   64 x 4 x 4000, 32 / 8 x 128                       52 / 70 / 57 (uncut, of which 3
//                                                     find the shares, 3 the join)
template <class Fit, class Body>
__device__ __forceinline__ void shared_units(const CacheAttention& a, Fit fit, Body body) {
  __shared__ int s_before[256], s_wave[5][4];  // what lies before a thread's (sequence, tile) pairs
  __shared__ Sequence s_first[256];            // its first sequence
  const int pairs = a.c.n_seqs * a.tiles, per = (pairs + 255) >> 8, heads = a.c.n_kv_heads;
  int mine = 0, most = 0, some = 0;  // blocks, the most of a pair, pairs with any
  for (int i = 0; i < per; ++i) {
    const int pair = (int)threadIdx.x * per + i;
    if (pair >= pairs) break;
    const int seq = over(pair, a.by_tiles);
    const Sequence s = sequence_of(a, seq);
    if (i == 0) s_first[threadIdx.x] = s;
    const int n = blocks_of(a, s, pair - seq * a.tiles);
    mine += n;
    most = max(most, n);
    some += n > 0;
  }
  // Units are cut into parts of at most `cut` blocks, of which a worker has `take`.
  int2 parts = sums_before(mine * heads, s_wave[0]);
  const int total = parts.y;
  int cut = 1, take = max(over(total + a.workers - 1, a.by_workers), a.least_share);
  if (a.units <= a.workers / 4 && per == 1) {
    // The least share, if its parts are no more than the workers, else one that is
    // sure to be.
    cut = take;
    take = 1;
    parts = sums_before((mine + cut - 1) / cut * heads, s_wave[1]);
    if (parts.y > a.workers) {
      cut = max((total + a.workers - a.units - 1) / (a.workers - a.units), a.least_share);
      parts = sums_before((mine + cut - 1) / cut * heads, s_wave[2]);
    }
  } else if (a.units <= a.workers && fit(take, most_of(most, s_wave[3]))) {
    cut = INT32_MAX >> 1;
    take = 1;
    parts = sums_before(some * heads, s_wave[4]);
  }
  s_before[threadIdx.x] = parts.x;
  __syncthreads();
  const int worker = worker_of((parts.y + take - 1) / take);
  if (worker < 0) return;
  int at = worker * take;
  const int end = min(at + take, parts.y);
  const int thread = last_upto(s_before, at);
  int start = uniform(s_before[thread]);
  Sequence s = uniform(s_first[thread]);
  // (A part of one unit has code of its own: what is in a loop over units is
  // scheduled for fewer registers, 3 to 7 % slower.)
  int pair = thread * per, seq = over(pair, a.by_tiles), tile = pair - seq * a.tiles;
  int n = 0, cuts = 0;
  while (true) {
    n = blocks_of(a, s, tile);
    cuts = (n + cut - 1) / cut;
    if (at < start + cuts * heads) break;
    start += cuts * heads;
    if (++tile == a.tiles) {
      tile = 0;
      s = uniform(sequence_of(a, ++seq));
    }
    ++pair;
  }
  int kvh = (at - start) / cuts;
  start += kvh * cuts;
  auto part_of = [&](int from, int to) {
    const int size = (n + cuts - 1) / cuts;
    Unit u = unit_of(a, s, seq, kvh, tile);
    u.whole = from == 0 && to == cuts;
    u.k0 = from * size << a.block_shift;
    u.k1 = min(to * size << a.block_shift, u.limit);
    u.slot = 2 * worker + (from == 0);
    if (to == cuts && threadIdx.x == 0)
      a.joins[pair * heads + kvh] = make_int2(u.whole ? -1 : start / take, worker);
    return u;
  };
  if (take == 1) {
    body(part_of(at - start, at - start + 1));
    return;
  }
  while (true) {
    const int to = min(cuts, end - start);
    body(part_of(at - start, to));
    at = start + to;
    if (at >= end) return;
    __syncthreads();  // LDS is read out
    start += cuts;
    if (++kvh < heads) continue;
    kvh = 0;
    do {
      ++pair;
      if (++tile == a.tiles) {
        tile = 0;
        s = uniform(sequence_of(a, ++seq));
      }
      n = cuts = blocks_of(a, s, tile);
    } while (n == 0);
  }
}

// The slot of part p of a unit that is joined: its first worker has its head,
// the others' first parts are its.
__device__ __forceinline__ int part_slot(int2 join, int p) { return 2 * (join.x + p) + (p == 0); }

// A lane's value combined with those of the lanes 16 and 32 apart.
template <class Op>
__device__ __forceinline__ float over_quarters(float v, Op op) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = op(__uint_as_float(r[0]), __uint_as_float(r[1]));
  const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return op(__uint_as_float(s[0]), __uint_as_float(s[1]));
}
__device__ __forceinline__ float max_of(float x, float y) { return fmaxf(x, y); }
__device__ __forceinline__ float sum_of(float x, float y) { return x + y; }

// What a lane holds of a block of 32 keys: the quarter lane / 16 of keys
// lane % 16 and 16 + lane % 16, and the byte of its scale.
template <int DH>
struct Block {
  Quarter<DH> k[2], v[2];
  uint32_t ks[2], vs[2];
  int bad;  // bit t: the table's entry of tile t is no page
};

// Pages of a wave's next 32 blocks, entry 2 j + t in that lane: tile t of 16
// keys of block block0 + step j.  -1: no page.
__device__ __forceinline__ int pages_ahead(const CacheAttention& a, int seq, int block0, int step, int k1) {
  const int lane = threadIdx.x & 63;
  const int key = (block0 + step * (lane >> 1)) * 32 + (lane & 1) * 16;
  if (key >= k1) return 0;
  const int page = a.c.table[(int64_t)seq * a.c.ld_table + (key >> a.c.page_shift)];
  return page >= 0 && page < a.c.n_pages ? page : -1;
}

template <int DH>
__device__ __forceinline__ void load_block(const CacheAttention& a, int64_t head_at, int pages, int entry,
                                           int key0, int lane, Block<DH>* b) {
  using L = PageLayout<DH>;
  const int quarter = lane >> 4;
  const int shift = a.c.page_shift, mask = (1 << shift) - 1;
  b->bad = 0;
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int page = __builtin_amdgcn_readlane(pages, entry + t);
    if (page < 0) b->bad |= 1 << t;
    const uint8_t* p = a.c.pages + max(page, 0) * a.c.page_bytes + head_at;
    // Tokens past the unit's keys are read too: they are in the page.
    const int slot = ((key0 + 16 * t) & mask) + (lane & 15);
    b->k[t].load(p + L::codes(shift, slot, 0) + quarter * (DH / 8));
    b->v[t].load(p + L::codes(shift, slot, 1) + quarter * (DH / 8));
    b->ks[t] = p[L::scales(shift, slot, 0) + quarter * L::SCALES / 4];
    b->vs[t] = p[L::scales(shift, slot, 1) + quarter * L::SCALES / 4];
  }
}

// The scales of a lane's quarters of key and value, as floats.  A key that is
// not there has small ones, so that nothing that stands in it is a NaN; one
// that has no page, or whose key or value is not finite, makes its score one.
__device__ __forceinline__ void scales_of(uint32_t ks, uint32_t vs, bool there, bool bad, float* k, float* v) {
  const bool nan = vs == NAN_SCALE || bad;
  *k = scale_of(!there ? 1u : nan ? NAN_SCALE : ks);
  *v = scale_of(!there || nan ? 1u : vs);
}

// Position of 16-byte chunk `chunk` of row `key` of V in LDS, rows of CPR chunks.
// The transposing reads take 32 bytes of eight consecutive rows at a time, which
// lie on different banks of the 64; a write takes one chunk of eight rows at a time,
// which lie on different ones of the 32 that it has (of 64 they did before: 8 cycles
// more for each write, 1 % of the time).
template <int CPR>
__device__ __forceinline__ uint32_t v_slot(int key, int chunk) {
  if constexpr (CPR == 16) return key * 16 + (chunk ^ ((key & 7) << 1 | (key >> 2 & 1)));
  if constexpr (CPR == 8) return key * 8 + (chunk ^ (key & 7));
  return key * 4 + (chunk ^ (key >> 1 & 3));
}

// Few rows: RT tiles of 16 against blocks of 32 keys, each of a unit's WAVES waves (4,
// or 1: the workgroup has four units) with blocks of its own.  Maxima and sums are a
// lane's own over its keys (a quarter of them) and joined at the end; so are the waves.
template <int DH, int RT, int WAVES>
__device__ __forceinline__ void few_rows_unit(const CacheAttention& a, const Unit& u) {
  constexpr int STEPS = DH / 32, FT = DH / 16, CPR = DH / 8;
  constexpr int STRIDE = DH + 4;  // floats of a staged output row
  constexpr int LDS_WAVE = (WAVES == 1 || 32 * DH * 2 > 16 * STRIDE * 4 ? 32 * DH * 2 : 16 * STRIDE * 4);
  __shared__ __attribute__((aligned(256))) uint8_t lds[(WAVES == 1 ? 1 : RT) * 4 * LDS_WAVE];
  const int lane = own_lane(), col = lane & 15, quarter = lane >> 4;
  const int own = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wave = WAVES == 1 ? 0 : own;
  const int G = a.group;

  // Every key waits for the table: it is asked for first.
  const int end = (u.k1 + 31) / 32;  // blocks
  int block = u.k0 / 32 + wave;
  int pages = block < end ? pages_ahead(a, u.seq, block, WAVES, u.k1) : 0;
  bf16x8 qf[RT][STEPS];
  int limit[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int row = min(u.row0 + rt * 16 + col, u.rows - 1);
    limit[rt] = row_limit(a, u, row);
    const int query = over(row, a.by_group);
    const uint16_t* q = a.q + (int64_t)(u.q_beg + query) * a.ld_q + (u.kvh * G + row - query * G) * DH;
#pragma unroll
    for (int kk = 0; kk < STEPS; ++kk)
      qf[rt][kk] = *reinterpret_cast<const bf16x8*>(q + quarter * (DH / 4) + kk * 8);
  }
  const int least = row_limit(a, u, u.row0);  // keys that every row sees

  float m_ref[RT], l_run[RT];
  f32x4 o[RT][FT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    m_ref[rt] = -FLT_MAX;
    l_run[rt] = 0.0f;
#pragma unroll
    for (int f = 0; f < FT; ++f) o[rt][f] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  }

  const int64_t head_at = u.kvh * PageLayout<DH>::head_bytes(a.c.page_shift);
  u32x4* const sv = reinterpret_cast<u32x4*>(lds + own * LDS_WAVE);
  int entry = 0;
  Block<DH> next;
  if (block < end) load_block<DH>(a, head_at, pages, 0, block * 32, lane, &next);
  for (; block < end; block += WAVES) {
    const Block<DH> b = next;
    if (block + WAVES < end) {
      entry += 2;
      if (entry == 64) {
        entry = 0;
        pages = pages_ahead(a, u.seq, block + WAVES, WAVES, u.k1);
      }
      load_block<DH>(a, head_at, pages, entry, (block + WAVES) * 32, lane, &next);
    }
    f32x4 s[RT][2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int key = block * 32 + 16 * t + col;
      float k_scale, v_scale;
      scales_of(b.ks[t], b.vs[t], key < u.k1, b.bad >> t & 1, &k_scale, &v_scale);
#pragma unroll
      for (int kk = 0; kk < STEPS; ++kk) {
        const bf16x8 k = decode8(b.k[t].w[kk], k_scale);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
          s[rt][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
              k, qf[rt][kk], kk == 0 ? f32x4{0.0f, 0.0f, 0.0f, 0.0f} : s[rt][t], 0, 0, 0);
        sv[v_slot<CPR>(16 * t + col, quarter * STEPS + kk)] =
            __builtin_bit_cast(u32x4, decode8(b.v[t].w[kk], v_scale));
      }
    }
    // V^T of feature tile f: keys 4 quarter .. + 3 and 16 further on, as the
    // scores' registers have them.  Half of the tiles are asked for before the
    // softmax and the others before the first half's products.
    auto v_fragment = [&](int f) {
      bf16x4 v[2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int key = 16 * t + 4 * quarter + (col >> 2);
        const uint32_t at = lds_address(sv) + v_slot<CPR>(key, 2 * f + (col >> 1 & 1)) * 16 + (col & 1) * 8;
        v[t] = __builtin_bit_cast(
            bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)at));
      }
      return __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7);
    };
    bf16x8 vf[FT];
#pragma unroll
    for (int f = 0; f < FT / 2; ++f) vf[f] = v_fragment(f);
    __builtin_amdgcn_sched_barrier(0);
    const bool some_hidden = block * 32 + 32 > least || block * 32 + 32 > u.k1;
    bf16x8 pb[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
#pragma unroll
      for (int i = 0; i < 8; ++i) s[rt][i >> 2][i & 3] *= a.scale_log2;
      if (some_hidden) {
        asm volatile("");  // a branch around the comparisons, not a selection by both
        const int seen = min(limit[rt], u.k1) - block * 32 - 4 * quarter;
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (16 * (i >> 2) + (i & 3) >= seen) s[rt][i >> 2][i & 3] = -INFINITY;
      }
      float most = s[rt][0][0];
#pragma unroll
      for (int i = 1; i < 8; ++i) most = fmaxf(most, s[rt][i >> 2][i & 3]);
      most = over_quarters(most, max_of);
      // The reference of the exponentials follows the maximum only where that
      // has grown by more than 2^8.
      if (__any(most > m_ref[rt] + 8.0f)) {
        const float m_new = fmaxf(m_ref[rt], most);
        const float alpha = __builtin_amdgcn_exp2f(m_ref[rt] - m_new);
        m_ref[rt] = m_new;
        l_run[rt] *= alpha;
#pragma unroll
        for (int f = 0; f < FT; ++f)
#pragma unroll
          for (int r = 0; r < 4; ++r) o[rt][f][r] *= alpha;
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float p = __builtin_amdgcn_exp2f(s[rt][i >> 2][i & 3] - m_ref[rt]);
        l_run[rt] += p;
        pb[rt][i] = (__bf16)p;
      }
    }
#pragma unroll
    for (int f = FT / 2; f < FT; ++f) vf[f] = v_fragment(f);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int f = 0; f < FT; ++f)
#pragma unroll
      for (int rt = 0; rt < RT; ++rt)
        o[rt][f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[f], pb[rt], o[rt][f], 0, 0, 0);
  }

  // Register r of tile f: feature 16 f + 4 quarter + r of row col.
  if constexpr (WAVES == 1) {
    // Through LDS, so that whole rows are stored, 16 bytes a lane.
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const float inv = 1.0f / over_quarters(l_run[rt], sum_of);
      const bool seen = min(limit[rt], u.k1) > u.k0;
#pragma unroll
      for (int f = 0; f < FT; ++f) {
        uint2 w;
        w.x = seen ? pack_bf16x2(o[rt][f][0] * inv, o[rt][f][1] * inv) : 0u;
        w.y = seen ? pack_bf16x2(o[rt][f][2] * inv, o[rt][f][3] * inv) : 0u;
        reinterpret_cast<uint2*>(sv + v_slot<CPR>(16 * rt + col, 2 * f + (quarter >> 1)))[quarter & 1] = w;
      }
    }
#pragma unroll
    for (int j = 0; j < RT * CPR / 4; ++j) {
      const int r = j * (64 / CPR) + lane / CPR, chunk = lane % CPR, row = u.row0 + r;
      const u32x4 w = sv[v_slot<CPR>(r, chunk)];
      if (row < u.rows) {
        const int query = over(row, a.by_group);
        *reinterpret_cast<u32x4*>(a.out + (int64_t)(u.q_beg + query) * a.ld_out + (u.kvh * G + row - query * G) * DH +
                                  chunk * 8) = w;
      }
    }
    return;
  }
  // The waves' parts are joined.
  __shared__ float s_m[WAVES][RT * 16], s_l[WAVES][RT * 16];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const float l = over_quarters(l_run[rt], sum_of);
    if (quarter == 0) {
      s_m[wave][rt * 16 + col] = m_ref[rt];
      s_l[wave][rt * 16 + col] = l;
    }
  }
  __syncthreads();
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    float m = s_m[0][rt * 16 + col];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) m = fmaxf(m, s_m[w][rt * 16 + col]);
    const float alpha = __builtin_amdgcn_exp2f(m_ref[rt] - m);
    float* const stage = reinterpret_cast<float*>(lds + (rt * WAVES + wave) * LDS_WAVE) + col * STRIDE + 4 * quarter;
#pragma unroll
    for (int f = 0; f < FT; ++f)
      *reinterpret_cast<f32x4*>(stage + 16 * f) =
          f32x4{o[rt][f][0] * alpha, o[rt][f][1] * alpha, o[rt][f][2] * alpha, o[rt][f][3] * alpha};
    __syncthreads();
    // Sixteen threads a row, four features each at a time.
    const int r = wave * 4 + quarter, row = u.row0 + rt * 16 + r;
    if (row < u.rows) {
      float ml = s_m[0][rt * 16 + r], l = 0.0f;
#pragma unroll
      for (int w = 1; w < WAVES; ++w) ml = fmaxf(ml, s_m[w][rt * 16 + r]);
#pragma unroll
      for (int w = 0; w < WAVES; ++w)
        l = fmaf(__builtin_amdgcn_exp2f(s_m[w][rt * 16 + r] - ml), s_l[w][rt * 16 + r], l);
      const bool seen = min(row_limit(a, u, row), u.k1) > u.k0;
      const float inv = seen ? 1.0f / l : 0.0f;
      for (int d = col * 4; d < DH; d += 64) {
        f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int w = 0; w < WAVES; ++w)
          v += *reinterpret_cast<const f32x4*>(lds + (rt * WAVES + w) * LDS_WAVE + (r * STRIDE + d) * 4);
        if (u.whole) {
          uint2 out;
          out.x = seen ? pack_bf16x2(v[0] * inv, v[1] * inv) : 0u;
          out.y = seen ? pack_bf16x2(v[2] * inv, v[3] * inv) : 0u;
          const int query = over(row, a.by_group);
          *reinterpret_cast<uint2*>(a.out + (int64_t)(u.q_beg + query) * a.ld_out +
                                    (u.kvh * G + row - query * G) * DH + d) = out;
        } else {
          const int64_t slot = (int64_t)u.slot * a.tile_rows + rt * 16 + r;
          *reinterpret_cast<f32x4*>(a.part_o + slot * DH + d) = v;
          if (d == 0) a.part_ml[slot] = make_float2(seen ? ml : -INFINITY, l);
        }
      }
    }
  }
}

// Many rows: four waves share blocks of 64 keys in LDS, decoded to bf16 by all of
// them, each wave a tile of 16 keys.  A block's codes are loaded two blocks ahead
// and decoded one ahead.  With GROUPS = 4 a wave has 32 rows against the whole block,
// with 2 against half of it, and the halves are joined in the end.
//
// Chunk c of row r is stored at c ^ f(r), so that neither the reads of K (a chunk
// of 16 of 32 rows at a time, on 64 banks), the transposing reads of V (64 bytes of
// four consecutive rows) nor the writes (a chunk of eight consecutive rows, on 32
// banks) have bank conflicts.  With r3 .. r0 the bits of r, f's are r1 ^ r3, r0, r1,
// r2 for rows of 16 chunks, r1, r2, r0 ^ r3 for 8 and r2, r1 ^ r3 for 4.
template <int CPR>
__device__ __forceinline__ uint32_t kv_position(int row, int chunk) {
  if constexpr (CPR == 16)
    return row * 16 + (chunk ^ (((row >> 1 ^ row >> 3) & 1) << 3 | (row & 1) << 2 | (row & 2) | (row >> 2 & 1)));
  if constexpr (CPR == 8) return row * 8 + (chunk ^ ((row & 2) << 1 | (row >> 1 & 2) | ((row ^ row >> 3) & 1)));
  return row * 4 + (chunk ^ ((row >> 1 & 3) ^ (row >> 3 & 1)));
}

__device__ __forceinline__ float over_halves(float v, float (*op)(float, float)) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return op(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

template <int DH, int GROUPS>
__device__ __forceinline__ void tile_unit(const CacheAttention& a, const Unit& u) {
  using L = PageLayout<DH>;
  constexpr int KSTEPS = DH / 16, DT = DH / 32, CPR = DH / 8, STEPS = DH / 32, KB = 64, T = GROUPS / 2;  // T: 32-key tiles of a wave
  constexpr uint32_t ROW = DH * 2, BUF = KB * ROW;
  __shared__ __attribute__((aligned(256))) u32x4 sKV[4 * BUF / 16];  // K blocks by parity, then V blocks
  const int lane = own_lane(), col = lane & 31, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int G = a.group;
  const int rows_of = wave % GROUPS, key_part = wave / GROUPS;
  const int row0 = u.row0 + rows_of * 32;
  const bool active = row0 < u.rows;  // a wave without rows still decodes
  const int row = min(row0 + col, u.rows - 1);
  const int limit = min(row_limit(a, u, row), u.k1);
  const int least = min(row_limit(a, u, min(row0, u.rows - 1)), u.k1);            // that every row sees
  const int most_keys = min(row_limit(a, u, min(row0 + 31, u.rows - 1)), u.k1);   // that some row sees

  const int64_t head_at = u.kvh * L::head_bytes(a.c.page_shift);
  const int shift = a.c.page_shift, mask = (1 << shift) - 1;
  const int n = (max(u.k1 - u.k0, 0) + KB - 1) / KB;
  // Pages of this wave's tile of blocks first .. first + 63.
  auto pages_from = [&](int first) {
    const int key = u.k0 + (first + lane) * KB + 16 * wave;
    if (key >= u.k1) return 0;
    const int page = a.c.table[(int64_t)u.seq * a.c.ld_table + (key >> shift)];
    return page >= 0 && page < a.c.n_pages ? page : -1;
  };
  int pages = n > 0 ? pages_from(0) : 0;
  bf16x8 qf[KSTEPS];
  const int query = over(row, a.by_group);
  const uint16_t* q = a.q + (int64_t)(u.q_beg + query) * a.ld_q + (u.kvh * G + row - query * G) * DH;
#pragma unroll
  for (int kk = 0; kk < KSTEPS; ++kk) qf[kk] = *reinterpret_cast<const bf16x8*>(q + (kk * 2 + half) * 8);

  Quarter<DH> raw_k, raw_v;
  uint32_t raw_ks = 0, raw_vs = 0;
  bool raw_bad = false;
  auto load = [&](int i) {
    if (i > 0 && (i & 63) == 0) pages = pages_from(i);
    const int page = __builtin_amdgcn_readlane(pages, i & 63);
    raw_bad = page < 0;
    const uint8_t* p = a.c.pages + max(page, 0) * a.c.page_bytes + head_at;
    const int slot = ((u.k0 + i * KB + 16 * wave) & mask) + (lane & 15), quarter = lane >> 4;
    raw_k.load(p + L::codes(shift, slot, 0) + quarter * (DH / 8));
    raw_v.load(p + L::codes(shift, slot, 1) + quarter * (DH / 8));
    raw_ks = p[L::scales(shift, slot, 0) + quarter * L::SCALES / 4];
    raw_vs = p[L::scales(shift, slot, 1) + quarter * L::SCALES / 4];
  };
  auto decode = [&](int i) {
    float k_scale, v_scale;
    const int r = 16 * wave + (lane & 15);
    scales_of(raw_ks, raw_vs, u.k0 + i * KB + r < u.k1, raw_bad, &k_scale, &v_scale);
    u32x4* const to = sKV + (i & 1) * (BUF / 16);
#pragma unroll
    for (int kk = 0; kk < STEPS; ++kk) {
      const uint32_t at = kv_position<CPR>(r, (lane >> 4) * STEPS + kk);
      to[at] = __builtin_bit_cast(u32x4, decode8(raw_k.w[kk], k_scale));
      to[2 * (BUF / 16) + at] = __builtin_bit_cast(u32x4, decode8(raw_v.w[kk], v_scale));
    }
  };

  const uint32_t lds = lds_address(sKV);
  const int tr_key = 4 * half + ((lane & 15) >> 2);
  const int tr_feat = 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
  uint32_t ka = lds + key_part * 32 * ROW + kv_position<CPR>(col, half) * 16u;
  uint32_t va = lds + key_part * 32 * ROW + 2 * BUF + kv_position<CPR>(tr_key, tr_feat >> 3) * 16u + (tr_feat & 7) * 2u;
  constexpr uint32_t H_SWZ = CPR == 16 ? 128 : 16;  // of 8 keys further on
  auto k_fragment = [&](int t, int kk) {
    return __builtin_bit_cast(
        bf16x8, *(const __attribute__((address_space(3))) u32x4*)((ka ^ kk * 32) + t * 32 * ROW));
  };
  auto v_fragment = [&](int c, int dt) {
    bf16x4 v[2];
#pragma unroll
    for (int h = 0; h < 2; ++h)
      v[h] = __builtin_bit_cast(
          bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)(
                      (va ^ (dt * 64 ^ h * H_SWZ)) + (16 * c + 8 * h) * ROW)));
    return __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7);
  };

  bool coarse = false;  // some row's maximum is 2^24 or more
  float m_ref = -FLT_MAX, l_run = 0.0f;
  f32x16 o[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[dt][r] = 0.0f;

  if (n > 0) {
    load(0);
    decode(0);
    if (n > 1) load(1);
  }
  for (int i = 0; i < n; ++i) {
    __syncthreads();  // the block is there, the other one read out
    auto next_block = [&] {
      if (i + 1 < n) {
        decode(i + 1);
        if (i + 2 < n) load(i + 2);
      }
    };
    const int key0 = u.k0 + i * KB + key_part * 32;
    if (active && key0 < most_keys) {
      f32x16 s[T];
#pragma unroll
      for (int t = 0; t < T; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) s[t][r] = 0.0f;
      // Ahead of the waves of the SIMD that are at their exponentials.
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int kk = 0; kk < KSTEPS; ++kk)
#pragma unroll
        for (int t = 0; t < T; ++t)
          s[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k_fragment(t, kk), qf[kk], s[t], 0, 0, 0);
      __builtin_amdgcn_s_setprio(0);
      next_block();
      // V^T of 16 keys is asked for ahead of the exponentials of the 16 before.
      bf16x8 vf[2][DT];
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) vf[0][dt] = v_fragment(0, dt);
      __builtin_amdgcn_sched_barrier(0);
      if (key0 + 32 * T > least) {
        asm volatile("");  // a branch around the comparisons, not a selection by both
        const int seen = limit - key0 - 4 * half;
#pragma unroll
        for (int r = 0; r < 16 * T; ++r)
          if (32 * (r >> 4) + 8 * (r >> 2 & 3) + (r & 3) >= seen) s[r >> 4][r & 15] = -INFINITY;
      }
      float most = s[0][0];
#pragma unroll
      for (int r = 1; r < 16 * T; ++r) most = fmaxf(most, s[r >> 4][r & 15]);
      most = over_halves(most, max_of) * a.scale_log2;
      if (__any(most > m_ref + 8.0f)) {
        const float m_new = fmaxf(m_ref, most);
        const float alpha = __builtin_amdgcn_exp2f(m_ref - m_new);
        m_ref = m_new;
        coarse = __any(fabsf(m_new) >= 0x1p24f);
        l_run *= alpha;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
          for (int r = 0; r < 16; ++r) o[dt][r] *= alpha;
      }
      // The reference is a rounded product, off from the exact ones of the
      // exponentials by up to half of its step: where that is large, the products
      // are rounded too.
      float factor = a.scale_log2;
      if (__builtin_expect(coarse, 0)) {
#pragma unroll
        for (int r = 0; r < 16 * T; ++r) s[r >> 4][r & 15] *= factor;
        factor = 1.0f;
      }
#pragma unroll
      for (int c = 0; c < 2 * T; ++c) {
        bf16x8 pb;
#pragma unroll
        for (int r = 0; r < 8; ++r) {
          const float p = __builtin_amdgcn_exp2f(fmaf(s[c >> 1][8 * (c & 1) + r], factor, -m_ref));
          l_run += p;
          pb[r] = (__bf16)p;
        }
        if (c + 1 < 2 * T) {
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) vf[c + 1 & 1][dt] = v_fragment(c + 1, dt);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
          o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[c & 1][dt], pb, o[dt], 0, 0, 0);
      }
    } else {
      next_block();
    }
    const uint32_t other = i & 1 ? 0u - BUF : BUF;
    ka += other;
    va += other;
  }
  l_run = over_halves(l_run, sum_of);
  const bool seen = limit > u.k0;
  __syncthreads();  // every wave has read its last block
  if constexpr (GROUPS == 2) {
    f32x4* const from = reinterpret_cast<f32x4*>(sKV) + rows_of * (32 * DH / 4) + lane;
    float2* const ml = reinterpret_cast<float2*>(sKV + 2 * (BUF / 16)) + rows_of * 64 + lane;
    if (key_part == 1) {
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int g = 0; g < 4; ++g)
          from[(dt * 4 + g) * 64] = f32x4{o[dt][4 * g], o[dt][4 * g + 1], o[dt][4 * g + 2], o[dt][4 * g + 3]};
      *ml = make_float2(m_ref, l_run);
    }
    __syncthreads();
    if (key_part == 1 || !active) return;
    const float2 other = *ml;
    const float m = fmaxf(m_ref, other.x);
    const float f = __builtin_amdgcn_exp2f(m_ref - m), g2 = __builtin_amdgcn_exp2f(other.x - m);
    m_ref = m;
    l_run = l_run * f + other.y * g2;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const f32x4 v = from[(dt * 4 + g) * 64];
#pragma unroll
        for (int r = 0; r < 4; ++r) o[dt][4 * g + r] = o[dt][4 * g + r] * f + v[r] * g2;
      }
  }
  if (!active) return;

  // Register r of tile dt: feature dt 32 + 8 (r / 4) + 4 half + r % 4 of row col.
  if (u.whole) {
    const float inv = 1.0f / l_run;
    // (Behind what the halves' join still reads and beside its maxima.)
    u32x4* const stage = sKV + (GROUPS == 2 ? 3 * (BUF / 16) : 0) + rows_of * (32 * CPR);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        uint2 w;
        w.x = seen ? pack_bf16x2(o[dt][4 * g] * inv, o[dt][4 * g + 1] * inv) : 0u;
        w.y = seen ? pack_bf16x2(o[dt][4 * g + 2] * inv, o[dt][4 * g + 3] * inv) : 0u;
        reinterpret_cast<uint2*>(stage + kv_position<CPR>(col, dt * 4 + g))[half] = w;
      }
    // Whole rows are stored, 16 bytes a lane.
#pragma unroll
    for (int j = 0; j < CPR / 2; ++j) {
      const int r = j * (64 / CPR) + lane / CPR, chunk = lane % CPR;
      const u32x4 w = stage[kv_position<CPR>(r, chunk)];
      if (row0 + r < u.rows) {
        const int query = over(row0 + r, a.by_group);
        __builtin_nontemporal_store(
            w, reinterpret_cast<u32x4*>(a.out + (int64_t)(u.q_beg + query) * a.ld_out +
                                        (u.kvh * G + row0 + r - query * G) * DH + chunk * 8));
      }
    }
    return;
  }
  if (row0 + col >= u.rows) return;
  const int64_t slot = (int64_t)u.slot * a.tile_rows + rows_of * 32 + col;
  if (half == 0) a.part_ml[slot] = make_float2(seen ? m_ref : -INFINITY, l_run);
  float* po = a.part_o + slot * DH;
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int g = 0; g < 4; ++g)
      *reinterpret_cast<float4*>(po + dt * 32 + g * 8 + half * 4) =
          make_float4(o[dt][4 * g], o[dt][4 * g + 1], o[dt][4 * g + 2], o[dt][4 * g + 3]);
}

template <int DH, int RT, bool SHARED>
__global__ __launch_bounds__(256)
__attribute__((amdgpu_waves_per_eu(PLACES[RT / 2][DH / 64]))) void few_rows_kernel(CacheAttention a) {
  auto body = [&](const Unit& u) { few_rows_unit<DH, RT, 4>(a, u); };
  // Half of the places of 16 rows stream as much as the memory gives; a join takes as
  // long as six blocks.
  auto fit = [](int share, int most) { return most <= share * (RT == 1 ? 2 : 1) + 6; };
  if constexpr (SHARED) shared_units(a, fit, body);
  else one_unit(a, blockIdx.x, body);
}

// A unit a wave.
template <int DH, int RT>
__global__ __launch_bounds__(256)
__attribute__((amdgpu_waves_per_eu(PLACES[RT / 2][DH / 64]))) void few_rows_wave_kernel(CacheAttention a) {
  const int index = (int)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (index < a.units) one_unit(a, index, [&](const Unit& u) { few_rows_unit<DH, RT, 1>(a, u); });
}

template <int DH, int GROUPS, bool SHARED>
__global__ __launch_bounds__(256)
__attribute__((amdgpu_waves_per_eu(SHARED ? PLACES[GROUPS / 2 + 1][DH / 64] : 2))) void tile_kernel(CacheAttention a) {
  auto body = [&](const Unit& u) { tile_unit<DH, GROUPS>(a, u); };
  auto fit = [](int, int) { return false; };  // (equal shares are as fast with even lengths)
  if constexpr (SHARED) shared_units(a, fit, body);
  else one_unit(a, blockIdx.x, body);
}

// The unit, and of a cut one the workers that have its parts, of a join.
struct Join {
  int seq, kvh, row0;
  int2 workers;
};
__device__ __forceinline__ Join join_of(const CacheAttention& a, int index) {
  const int pair = over(index, a.by_heads), seq = over(pair, a.by_tiles);
  return {seq, index - pair * a.c.n_kv_heads, (pair - seq * a.tiles) * a.tile_rows, a.joins[index]};  // (without rows whatever stands there)
}

// Joins the parts of units that few workers have: eight rows a wave, 16 bytes a
// lane, BATCH parts loaded together.
template <int DH, int BATCH>
__global__ __launch_bounds__(256) void join_rows_kernel(CacheAttention a, int row_groups) {
  constexpr int LANES = DH / 4, STEP = 64 / LANES, N = 8 / STEP;  // of a row; rows at a time
  const int lane = threadIdx.x & 63;
  const int index = (int)(blockIdx.x / (unsigned)row_groups);
  const int r0 = (int)(blockIdx.x % (unsigned)row_groups) * 32 + (int)(threadIdx.x >> 6) * 8 + lane / LANES;
  const Join j = join_of(a, index);
  const Sequence s = uniform(sequence_of(a, j.seq));
  const int rows = min(a.tile_rows, s.rows - j.row0);
  if (rows <= 0 || j.workers.x < 0) return;
  const int parts = j.workers.y - j.workers.x + 1;
  float m[N], l[N];
  f32x4 o[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    m[i] = -INFINITY;
    l[i] = 0.0f;
    o[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  }
  for (int p0 = 0; p0 < parts; p0 += BATCH) {
    float2 ml[BATCH][N];
    f32x4 v[BATCH][N];
#pragma unroll
    for (int q = 0; q < BATCH; ++q) {
      const int64_t slot = (int64_t)part_slot(j.workers, min(p0 + q, parts - 1)) * a.tile_rows;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int64_t row = slot + min(r0 + i * STEP, rows - 1);
        ml[q][i] = a.part_ml[row];
        v[q][i] = *reinterpret_cast<const f32x4*>(a.part_o + row * DH + lane % LANES * 4);
      }
    }
#pragma unroll
    for (int q = 0; q < BATCH; ++q)
#pragma unroll
      for (int i = 0; i < N; ++i) {
        if (p0 + q >= parts || ml[q][i].x == -INFINITY) continue;  // (no key for the row in it: zeros)
        const float top = fmaxf(m[i], ml[q][i].x);
        const float f = __builtin_amdgcn_exp2f(m[i] - top), g = __builtin_amdgcn_exp2f(ml[q][i].x - top);
        m[i] = top;
        l[i] = l[i] * f + ml[q][i].y * g;
#pragma unroll
        for (int d = 0; d < 4; ++d) o[i][d] = o[i][d] * f + v[q][i][d] * g;
      }
  }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int r = r0 + i * STEP, row = j.row0 + r;
    if (r >= rows) continue;
    const float inv = m[i] > -INFINITY ? 1.0f / l[i] : 0.0f;
    const int query = over(row, a.by_group), G = a.group;
    uint2 w;
    w.x = pack_bf16x2(o[i][0] * inv, o[i][1] * inv);
    w.y = pack_bf16x2(o[i][2] * inv, o[i][3] * inv);
    *reinterpret_cast<uint2*>(a.out + (int64_t)(s.q_beg + query) * a.ld_out + (j.kvh * G + row - query * G) * DH +
                              lane % LANES * 4) = w;
  }
}

// Joins the parts of a row that many workers have: WAVES waves take parts w, w +
// WAVES, ..., BATCH of them loaded together, and are added in order.
template <int DH, int WAVES, int BATCH>
__global__ __launch_bounds__(64 * WAVES) void join_kernel(CacheAttention a, int rows_each) {
  constexpr int PER = DH < 64 ? 1 : DH / 64;
  __shared__ float sm[WAVES], so[WAVES][DH + 1];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int index = (int)(blockIdx.x / (unsigned)rows_each), r = (int)(blockIdx.x % (unsigned)rows_each);
  const Join j = join_of(a, index);
  const Sequence s = uniform(sequence_of(a, j.seq));
  const int row = j.row0 + r;
  if (row >= s.rows || r >= a.tile_rows || j.workers.x < 0) return;
  const int parts = j.workers.y - j.workers.x + 1;
  float m = -INFINITY, l = 0.0f, o[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) o[i] = 0.0f;
  for (int p0 = wave; p0 < parts; p0 += WAVES * BATCH) {
    float2 ml[BATCH];
    float v[BATCH][PER];
#pragma unroll
    for (int q = 0; q < BATCH; ++q) {
      const int64_t s = (int64_t)part_slot(j.workers, min(p0 + q * WAVES, parts - 1)) * a.tile_rows + r;
      ml[q] = a.part_ml[s];
#pragma unroll
      for (int i = 0; i < PER; ++i) v[q][i] = lane < DH ? a.part_o[s * DH + lane * PER + i] : 0.0f;
    }
    float m_new = m;
#pragma unroll
    for (int q = 0; q < BATCH; ++q)
      if (p0 + q * WAVES < parts) m_new = fmaxf(m_new, ml[q].x);
    if (m_new == -INFINITY) continue;  // no key for the row so far: nothing but zeros
    const float alpha = __builtin_amdgcn_exp2f(m - m_new);
    m = m_new;
    l *= alpha;
#pragma unroll
    for (int i = 0; i < PER; ++i) o[i] *= alpha;
#pragma unroll
    for (int q = 0; q < BATCH; ++q) {
      const bool on = p0 + q * WAVES < parts;
      const float f = on ? __builtin_amdgcn_exp2f(ml[q].x - m) : 0.0f;
      l = fmaf(f, on ? ml[q].y : 0.0f, l);
#pragma unroll
      for (int i = 0; i < PER; ++i) o[i] = fmaf(f, on ? v[q][i] : 0.0f, o[i]);
    }
  }
  if (lane == 0) {
    sm[wave] = m;
    so[wave][DH] = l;
  }
  if (lane < DH)
#pragma unroll
    for (int i = 0; i < PER; ++i) so[wave][lane * PER + i] = o[i];
  __syncthreads();
  if (wave > 0) return;
  m = sm[0];
#pragma unroll
  for (int w = 1; w < WAVES; ++w) m = fmaxf(m, sm[w]);
  l = 0.0f;
#pragma unroll
  for (int i = 0; i < PER; ++i) o[i] = 0.0f;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) {
    const float f = m > -INFINITY ? __builtin_amdgcn_exp2f(sm[w] - m) : 0.0f;
    l = fmaf(f, so[w][DH], l);
#pragma unroll
    for (int i = 0; i < PER; ++i)
      if (lane < DH) o[i] = fmaf(f, so[w][lane * PER + i], o[i]);
  }
  const float inv = m > -INFINITY ? 1.0f / l : 0.0f;
  const int query = over(row, a.by_group), G = a.group;
  uint16_t* out = a.out + (int64_t)(s.q_beg + query) * a.ld_out + (j.kvh * G + row - query * G) * DH;
  if constexpr (PER == 2)
    reinterpret_cast<uint32_t*>(out)[lane] = pack_bf16x2(o[0] * inv, o[1] * inv);
  else if (lane < DH)
    out[lane] = (uint16_t)(pack_bf16x2(o[0] * inv, 0.0f) & 0xffffu);
}

template <int DH>
hipError_t launch(const CacheAttention& a, hipStream_t stream) {
  const dim3 grid(a.workers ? a.workers : a.units), block(256);
  if (a.wave_units) {
    const dim3 fours((a.units + 3) / 4);
    if (a.tile_rows == 16) hipLaunchKernelGGL((few_rows_wave_kernel<DH, 1>), fours, block, 0, stream, a);
    else hipLaunchKernelGGL((few_rows_wave_kernel<DH, 2>), fours, block, 0, stream, a);
    return hipGetLastError();
  }
#define SURGE_LAUNCH(...)                                                                  \
  do {                                                                                     \
    if (a.workers)                                                                         \
      hipLaunchKernelGGL((__VA_ARGS__, true>), grid, block, 0, stream, a);                 \
    else                                                                                   \
      hipLaunchKernelGGL((__VA_ARGS__, false>), grid, block, 0, stream, a);                \
  } while (0)
  if (a.tile_rows == 16) SURGE_LAUNCH(few_rows_kernel<DH, 1);
  if (a.tile_rows == 32) SURGE_LAUNCH(few_rows_kernel<DH, 2);
  if (a.tile_rows == 64) SURGE_LAUNCH(tile_kernel<DH, 2);
  if (a.tile_rows == 128) SURGE_LAUNCH(tile_kernel<DH, 4);
#undef SURGE_LAUNCH
  if (a.workers == 0) return hipGetLastError();
  const int rows = (int)std::min<int64_t>(a.tile_rows, (int64_t)a.max_rows * a.group);
  if (a.join_waves == 16) {
    hipLaunchKernelGGL((join_kernel<DH, 16, 8>), dim3(a.units * rows), dim3(1024), 0, stream, a, rows);
  } else if (a.join_waves == 4) {
    hipLaunchKernelGGL((join_kernel<DH, 4, 8>), dim3(a.units * rows), dim3(256), 0, stream, a, rows);
  } else if (a.join_waves == 1) {
    hipLaunchKernelGGL((join_kernel<DH, 1, 4>), dim3(a.units * rows), dim3(64), 0, stream, a, rows);
  } else {
    const int groups = (rows + 31) / 32;
    hipLaunchKernelGGL((join_rows_kernel<DH, 3>), dim3(a.units * groups), dim3(256), 0, stream, a, groups);
  }
  return hipGetLastError();
}

}  // namespace

Divisor divisor(int d) {
  int s = 0;
  while ((1ll << s) < d) ++s;
  return {(uint32_t)(((1ull << (31 + s)) + d - 1) / d), s};
}

hipError_t launch_cache_attention(const CacheAttention& a, int d_head, hipStream_t stream) {
  if (d_head == 32) return launch<32>(a, stream);
  if (d_head == 64) return launch<64>(a, stream);
  return launch<128>(a, stream);
}

}  // namespace surge
