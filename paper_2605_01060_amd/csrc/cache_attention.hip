// Attention over a cache in 4 bits (gfx950, bf16 MFMA, fp32 softmax).
//
//   out[t, h] = sum_k p_k V[k, h / G] / sum_k p_k,
//   p_k = exp(scale Q[t, h] . K[k, h / G]) over the positions that row t sees,
//
// G = heads per key head; a row that sees none gives zeros.  The G query heads
// that share a key head are rows of one matrix: row r of (sequence, key head)
// is query r / G, head r % G of the group.
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

// A unit's rows and keys, from the device's offsets and lengths.
struct Unit {
  int64_t seq;
  int tile, kvh, split;
  int q_beg, rows;       // first query row of the sequence, rows of its tiles
  int row0, first, last; // of the tile; first: position that row 0 of the sequence is at
  int k0, k1;            // keys of the unit
  int limit;             // keys that the tile's last row sees
  int slot;
};

// Keys that a row sees.
__device__ __forceinline__ int row_limit(const CacheAttention& a, const Unit& u, int row) {
  return a.causal ? u.first + row / a.group + 1 : u.limit;
}

__device__ __forceinline__ bool unit_of(const CacheAttention& a, int64_t index, Unit* u) {
  u->split = (int)(index % a.splits);
  index /= a.splits;
  u->kvh = (int)(index % a.c.n_kv_heads);
  index /= a.c.n_kv_heads;
  u->seq = index % a.c.n_seqs;
  u->tile = a.tiles - 1 - (int)(index / a.c.n_seqs);  // the last rows see the most keys
  int beg, n;
  if (a.r.cu) {
    beg = min(max(a.r.cu[u->seq], 0), a.r.n_rows);
    n = min(max(a.r.cu[u->seq + 1], beg), a.r.n_rows) - beg;
  } else {
    beg = (int)u->seq * a.r.each;
    n = a.r.each;
  }
  const int length = length_of(a.c, (int)u->seq);
  u->q_beg = beg;
  u->first = length - n;
  u->rows = min(n, a.max_rows) * a.group;
  u->row0 = u->tile * a.tile_rows;
  if (u->row0 >= u->rows) return false;
  const int last = min(u->row0 + a.tile_rows, u->rows) - 1;
  u->limit = a.causal ? max(u->first + last / a.group + 1, 0) : length;
  u->k0 = u->split * a.chunk;
  u->k1 = min(u->k0 + a.chunk, u->limit);
  if (u->split > 0 && u->k0 >= u->limit) return false;
  u->slot = (int)(((u->seq * a.tiles + u->tile) * a.c.n_kv_heads + u->kvh) * a.splits + u->split);
  return true;
}

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
__device__ __forceinline__ int pages_ahead(const CacheAttention& a, int64_t seq, int block0, int step, int k1) {
  const int lane = threadIdx.x & 63;
  const int key = (block0 + step * (lane >> 1)) * 32 + (lane & 1) * 16;
  if (key >= k1) return 0;
  const int page = a.c.table[seq * a.c.ld_table + (key >> a.c.page_shift)];
  return page >= 0 && page < a.c.n_pages ? page : -1;
}

template <int DH>
__device__ __forceinline__ void load_block(const CacheAttention& a, int64_t head_at, int pages, int entry,
                                           int key0, int k1, Block<DH>* b) {
  using L = PageLayout<DH>;
  const int lane = threadIdx.x & 63, quarter = lane >> 4;
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

// Position of 16-byte chunk `chunk` of row `key` of V in LDS, rows of CPR
// chunks: the transposing reads take 32 bytes of eight consecutive rows at a
// time and the writes one chunk of sixteen, neither with a bank conflict at
// d_head 64 and 128 (two-way in a part of the writes at 32).
template <int CPR>
__device__ __forceinline__ uint32_t v_slot(int key, int chunk) {
  if constexpr (CPR == 16) return key * 16 + (chunk ^ ((key & 7) << 1 | (key >> 3 & 1)));
  if constexpr (CPR == 8) return key * 8 + (chunk ^ ((key >> 1 & 3) << 1 | (key >> 3 & 1)));
  return key * 4 + (chunk ^ (key >> 2 & 1) * 3);
}

// Few rows: RT tiles of 16 against blocks of 32 keys, each wave of four with
// blocks of its own.
template <int DH, int RT>
__global__ __launch_bounds__(256) void few_rows_kernel(CacheAttention a) {
  constexpr int STEPS = DH / 32, FT = DH / 16, CPR = DH / 8, WAVES = 4;
  constexpr int STRIDE = DH + 4;  // floats of a staged output row
  constexpr int LDS_WAVE = (32 * DH * 2 > 16 * STRIDE * 4 ? 32 * DH * 2 : 16 * STRIDE * 4);
  __shared__ __attribute__((aligned(256))) uint8_t lds[WAVES * LDS_WAVE];
  __shared__ float s_m[WAVES][RT * 16], s_l[WAVES][RT * 16];
  Unit u;
  if (!unit_of(a, blockIdx.x, &u)) return;
  const int lane = threadIdx.x & 63, col = lane & 15, quarter = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int G = a.group;

  bf16x8 qf[RT][STEPS];
  int limit[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int row = min(u.row0 + rt * 16 + col, u.rows - 1);
    limit[rt] = row_limit(a, u, row);
    const uint16_t* q = a.q + (int64_t)(u.q_beg + row / G) * a.ld_q + (u.kvh * G + row % G) * DH;
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
  u32x4* const sv = reinterpret_cast<u32x4*>(lds + wave * LDS_WAVE);
  const int end = (u.k1 + 31) / 32;  // blocks
  int block = u.k0 / 32 + wave;
  int pages = 0, entry = 0;
  Block<DH> next;
  if (block < end) {
    pages = pages_ahead(a, u.seq, block, WAVES, u.k1);
    load_block<DH>(a, head_at, pages, 0, block * 32, u.k1, &next);
  }
  for (; block < end; block += WAVES) {
    const Block<DH> b = next;
    if (block + WAVES < end) {
      entry += 2;
      if (entry == 64) {
        entry = 0;
        pages = pages_ahead(a, u.seq, block + WAVES, WAVES, u.k1);
      }
      load_block<DH>(a, head_at, pages, entry, (block + WAVES) * 32, u.k1, &next);
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
    const bool some_hidden = block * 32 + 32 > least || block * 32 + 32 > u.k1;
    bf16x8 pb[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const int seen = min(limit[rt], u.k1) - block * 32 - 4 * quarter;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          s[rt][t][r] *= a.scale_log2;
          if (some_hidden && 16 * t + r >= seen) s[rt][t][r] = -INFINITY;
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
    // V^T of feature tile f: keys 4 quarter .. + 3 and 16 further on, as the
    // scores' registers have them.
#pragma unroll
    for (int f = 0; f < FT; ++f) {
      bf16x4 v[2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int key = 16 * t + 4 * quarter + (col >> 2);
        const uint32_t at = lds_address(sv) + v_slot<CPR>(key, 2 * f + (col >> 1 & 1)) * 16 + (col & 1) * 8;
        v[t] = __builtin_bit_cast(
            bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)at));
      }
      const bf16x8 vf = __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
      for (int rt = 0; rt < RT; ++rt)
        o[rt][f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pb[rt], o[rt][f], 0, 0, 0);
    }
  }

  // The waves' parts are joined.  Register r of tile f: feature 16 f + 4
  // quarter + r of row col.
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const float l = over_quarters(l_run[rt], sum_of);
    if (quarter == 0) {
      s_m[wave][rt * 16 + col] = m_ref[rt];
      s_l[wave][rt * 16 + col] = l;
    }
  }
  __syncthreads();
  const bool whole = a.splits == 1 || u.limit <= a.chunk;
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    float m = s_m[0][rt * 16 + col];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) m = fmaxf(m, s_m[w][rt * 16 + col]);
    const float alpha = __builtin_amdgcn_exp2f(m_ref[rt] - m);
    float* const stage = reinterpret_cast<float*>(lds + wave * LDS_WAVE) + col * STRIDE + 4 * quarter;
#pragma unroll
    for (int f = 0; f < FT; ++f)
      *reinterpret_cast<f32x4*>(stage + 16 * f) =
          f32x4{o[rt][f][0] * alpha, o[rt][f][1] * alpha, o[rt][f][2] * alpha, o[rt][f][3] * alpha};
    __syncthreads();
    // Sixteen threads a row, four features each at a time.
    const int r = threadIdx.x >> 4, row = u.row0 + rt * 16 + r;
    if (row < u.rows) {
      float ml = s_m[0][rt * 16 + r], l = 0.0f;
#pragma unroll
      for (int w = 1; w < WAVES; ++w) ml = fmaxf(ml, s_m[w][rt * 16 + r]);
#pragma unroll
      for (int w = 0; w < WAVES; ++w)
        l = fmaf(__builtin_amdgcn_exp2f(s_m[w][rt * 16 + r] - ml), s_l[w][rt * 16 + r], l);
      const bool seen = min(row_limit(a, u, row), u.k1) > u.k0;
      const float inv = seen ? 1.0f / l : 0.0f;
      for (int d = (threadIdx.x & 15) * 4; d < DH; d += 64) {
        f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int w = 0; w < WAVES; ++w)
          v += *reinterpret_cast<const f32x4*>(lds + w * LDS_WAVE + (r * STRIDE + d) * 4);
        if (whole) {
          uint2 out;
          out.x = seen ? pack_bf16x2(v[0] * inv, v[1] * inv) : 0u;
          out.y = seen ? pack_bf16x2(v[2] * inv, v[3] * inv) : 0u;
          *reinterpret_cast<uint2*>(a.out + (int64_t)(u.q_beg + row / G) * a.ld_out +
                                    (u.kvh * G + row % G) * DH + d) = out;
        } else {
          const int64_t slot = (int64_t)u.slot * a.tile_rows + rt * 16 + r;
          *reinterpret_cast<f32x4*>(a.part_o + slot * DH + d) = v;
          if (d == 0) a.part_ml[slot] = make_float2(seen ? ml : -INFINITY, l);
        }
      }
    }
    __syncthreads();
  }
}

// Many rows: four waves of 32 share blocks of 64 keys in LDS, decoded to bf16 by
// all of them, each wave a tile of 16 keys.  A block's codes are loaded two blocks
// ahead and decoded one ahead.
//
// Chunk c of row r is stored at c ^ f(r), so that neither the reads of K (a chunk
// of 32 rows), the transposing reads of V (64 bytes of four consecutive rows) nor,
// at d_head 128, the writes (a chunk of 16 rows) have bank conflicts.
template <int CPR>
__device__ __forceinline__ uint32_t kv_position(int row, int chunk) {
  if constexpr (CPR == 16) return row * 16 + (chunk ^ ((row & 3) << 2 | (row >> 2 & 3)));
  if constexpr (CPR == 8) return row * 8 + (chunk ^ ((row >> 1 & 1) << 2 | (row >> 2 & 3)));
  return swz<4>(row, chunk);
}

__device__ __forceinline__ float over_halves(float v, float (*op)(float, float)) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return op(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

template <int DH>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2))) void tile_kernel(CacheAttention a) {
  using L = PageLayout<DH>;
  constexpr int KSTEPS = DH / 16, DT = DH / 32, CPR = DH / 8, STEPS = DH / 32, KB = 64, T = KB / 32;
  constexpr uint32_t ROW = DH * 2, BUF = KB * ROW;
  __shared__ __attribute__((aligned(256))) u32x4 sKV[4 * BUF / 16];  // K blocks by parity, then V blocks
  Unit u;
  if (!unit_of(a, blockIdx.x, &u)) return;
  const int lane = threadIdx.x & 63, col = lane & 31, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int G = a.group;
  const int row0 = u.row0 + wave * 32;
  const bool active = row0 < u.rows;  // a wave without rows still decodes
  const int row = min(row0 + col, u.rows - 1);
  const int limit = min(row_limit(a, u, row), u.k1);
  const int least = min(row_limit(a, u, min(row0, u.rows - 1)), u.k1);            // that every row sees
  const int most_keys = min(row_limit(a, u, min(row0 + 31, u.rows - 1)), u.k1);   // that some row sees

  bf16x8 qf[KSTEPS];
  const uint16_t* q = a.q + (int64_t)(u.q_beg + row / G) * a.ld_q + (u.kvh * G + row % G) * DH;
#pragma unroll
  for (int kk = 0; kk < KSTEPS; ++kk) qf[kk] = *reinterpret_cast<const bf16x8*>(q + (kk * 2 + half) * 8);

  const int64_t head_at = u.kvh * L::head_bytes(a.c.page_shift);
  const int shift = a.c.page_shift, mask = (1 << shift) - 1;
  const int n = (max(u.k1 - u.k0, 0) + KB - 1) / KB;
  // Pages of this wave's tile of blocks first .. first + 63.
  auto pages_from = [&](int first) {
    const int key = u.k0 + (first + lane) * KB + 16 * wave;
    if (key >= u.k1) return 0;
    const int page = a.c.table[u.seq * a.c.ld_table + (key >> shift)];
    return page >= 0 && page < a.c.n_pages ? page : -1;
  };
  int pages = n > 0 ? pages_from(0) : 0;
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
  uint32_t ka = lds + kv_position<CPR>(col, half) * 16u;
  uint32_t va = lds + 2 * BUF + kv_position<CPR>(tr_key, tr_feat >> 3) * 16u + (tr_feat & 7) * 2u;
  constexpr uint32_t H_SWZ = CPR == 4 ? 16 : 32;  // of 8 keys further on
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
    if (i + 1 < n) {
      decode(i + 1);
      if (i + 2 < n) load(i + 2);
    }
    const int key0 = u.k0 + i * KB;
    if (active && key0 < most_keys) {
      f32x16 s[T];
#pragma unroll
      for (int t = 0; t < T; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) s[t][r] = 0.0f;
#pragma unroll
      for (int kk = 0; kk < KSTEPS; ++kk)
#pragma unroll
        for (int t = 0; t < T; ++t)
          s[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k_fragment(t, kk), qf[kk], s[t], 0, 0, 0);
      if (key0 + KB > least) {
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
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
          o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v_fragment(c, dt), pb, o[dt], 0, 0, 0);
      }
    }
    const uint32_t other = i & 1 ? 0u - BUF : BUF;
    ka += other;
    va += other;
  }
  l_run = over_halves(l_run, sum_of);
  const bool seen = limit > u.k0;

  // Register r of tile dt: feature dt 32 + 8 (r / 4) + 4 half + r % 4 of row col.
  if (a.splits == 1 || u.limit <= a.chunk) {
    __syncthreads();  // every wave has read its last block
    if (!active) return;
    const float inv = 1.0f / l_run;
    u32x4* stage = sKV + wave * (32 * CPR);
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
      if (row0 + r < u.rows)
        __builtin_nontemporal_store(
            w, reinterpret_cast<u32x4*>(a.out + (int64_t)(u.q_beg + (row0 + r) / G) * a.ld_out +
                                        (u.kvh * G + (row0 + r) % G) * DH + chunk * 8));
    }
    return;
  }
  if (row0 + col >= u.rows) return;
  const int64_t slot = (int64_t)u.slot * a.tile_rows + wave * 32 + col;
  if (half == 0) a.part_ml[slot] = make_float2(seen ? m_ref : -INFINITY, l_run);
  float* po = a.part_o + slot * DH;
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int g = 0; g < 4; ++g)
      *reinterpret_cast<float4*>(po + dt * 32 + g * 8 + half * 4) =
          make_float4(o[dt][4 * g], o[dt][4 * g + 1], o[dt][4 * g + 2], o[dt][4 * g + 3]);
}

// Joins the parts of a row of one key head: a wave a row, in the order of the
// keys.
template <int DH>
__global__ __launch_bounds__(256) void join_kernel(CacheAttention a) {
  constexpr int PER = DH < 64 ? 1 : DH / 64;
  const int lane = threadIdx.x & 63;
  const int64_t wave = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = (int)(wave % a.tile_rows);
  Unit u;
  if (!unit_of(a, wave / a.tile_rows * a.splits, &u)) return;
  const int row = u.row0 + r;
  if (u.limit <= a.chunk || row >= u.rows) return;
  const int parts = (u.limit + a.chunk - 1) / a.chunk;
  auto slot = [&](int p) { return (int64_t)(u.slot + p) * a.tile_rows + r; };
  float m = -INFINITY;
  for (int p = lane; p < parts; p += 64) m = fmaxf(m, a.part_ml[slot(p)].x);
  m = wave_max(m);
  float l = 0.0f, o[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) o[i] = 0.0f;
  // Without any key for the row every part is zeros: nothing to add.
#pragma unroll 4
  for (int p = 0; p < (m > -INFINITY ? parts : 0); ++p) {
    const float2 ml = a.part_ml[slot(p)];
    const float f = __builtin_amdgcn_exp2f(ml.x - m);
    l = fmaf(f, ml.y, l);
#pragma unroll
    for (int i = 0; i < PER; ++i)
      if (lane < DH) o[i] = fmaf(f, a.part_o[slot(p) * DH + lane * PER + i], o[i]);
  }
  const float inv = m > -INFINITY ? 1.0f / l : 0.0f;
  const int G = a.group;
  uint16_t* out = a.out + (int64_t)(u.q_beg + row / G) * a.ld_out + (u.kvh * G + row % G) * DH;
  if constexpr (PER == 2)
    reinterpret_cast<uint32_t*>(out)[lane] = pack_bf16x2(o[0] * inv, o[1] * inv);
  else if (lane < DH)
    out[lane] = (uint16_t)(pack_bf16x2(o[0] * inv, 0.0f) & 0xffffu);
}

template <int DH>
hipError_t launch(const CacheAttention& a, hipStream_t stream) {
  const int64_t tiles = (int64_t)a.tiles * a.c.n_seqs * a.c.n_kv_heads;
  const dim3 grid((unsigned)(tiles * a.splits)), block(256);
  if (a.tile_rows == 16) hipLaunchKernelGGL((few_rows_kernel<DH, 1>), grid, block, 0, stream, a);
  if (a.tile_rows == 32) hipLaunchKernelGGL((few_rows_kernel<DH, 2>), grid, block, 0, stream, a);
  if (a.tile_rows == 64) hipLaunchKernelGGL((few_rows_kernel<DH, 4>), grid, block, 0, stream, a);
  if (a.tile_rows == 128) hipLaunchKernelGGL(tile_kernel<DH>, grid, block, 0, stream, a);
  if (a.splits > 1)
    hipLaunchKernelGGL(join_kernel<DH>, dim3((unsigned)(tiles * a.tile_rows / 4)), block, 0, stream, a);
  return hipGetLastError();
}

}  // namespace

CacheShape cache_attention_shape(int64_t n_seqs, int64_t max_rows, int n_kv_heads, int group, int d_head,
                                 int64_t max_length, int n_cus) {
  CacheShape s;
  const int64_t rows = max_rows * group;
  s.tile_rows = rows <= 16 ? 16 : rows <= 32 ? 32 : rows <= 64 ? 64 : 128;
  s.tiles = (rows + s.tile_rows - 1) / s.tile_rows;
  const int64_t units = n_seqs * n_kv_heads * s.tiles;
  const int64_t want = std::max<int64_t>(1, 4 * (int64_t)n_cus / units);
  // Whole rounds of blocks of the four waves.
  s.chunk = std::max<int64_t>(256, ((max_length + want - 1) / want + 127) / 128 * 128);
  s.splits = std::max<int64_t>(1, (max_length + s.chunk - 1) / s.chunk);
  return s;
}

hipError_t launch_cache_attention(const CacheAttention& a, int d_head, hipStream_t stream) {
  if (d_head == 32) return launch<32>(a, stream);
  if (d_head == 64) return launch<64>(a, stream);
  return launch<128>(a, stream);
}

}  // namespace surge
