// Cross attention (gfx950, bf16 MFMA, fp32 softmax): the queries of each
// sequence attend to the states of its text, whose number is another one.
//
//   out[t, h] = sum_k p_k V[k, h / G] / sum_k p_k,
//   p_k = exp(scale Q[t, h] . K[k, h / G]) over the text's unmasked keys,
//
// G = heads per key head.  A sequence without (unmasked) keys gives zeros.
//
// The G query heads that share a key head are rows of one matrix: row r of
// (sequence, key head) is query r / G, head r % G of the group, so that a
// step of one query with shared heads fills a tile as G queries would.
//
// A unit is up to 128 rows of one (sequence, key head) over a range of its
// keys, in waves of 32 rows that share blocks of keys in LDS.  A wave computes
// S^T = K Q^T with 32x32x16 MFMAs, so that a lane owns one row (running
// maximum, sum and rescaling are the lane's own, joined with lane ^ 32 that
// has the other half of a key block), keeps the probabilities in registers as
// the operand of O^T += V^T P^T, and reads V^T from the row-major V block with
// the transposing LDS read.  The probabilities are rounded to bf16, the type
// of V and of the MFMA; maxima, sums and outputs stay fp32.  Where one
// (sequence, key head)'s keys are split over units, each writes its maximum,
// sum and unnormalised output in fp32, and a second kernel joins them in key
// order.
//
// Unit sizes: 128 rows against 64 keys (a key block is read from LDS once for
// four waves' rows), 64 rows against 32 keys for sequences of 33 to 64 rows
// (2000 texts of 64 keys, 64 queries, 12 x 64: 225 us as half-empty units of
// 128, 187 so) and one wave of 32 rows against 32 keys, with the most waves
// per CU, for fewer (a stream of keys).
//
// At d_head 128 the registers of 128 rows against 64 keys let a CU have two such
// units, against 32 keys three, whose exponentials cover more of the others'
// MFMAs; a block of 64 keys is the shorter chain.  The plan takes 32 where units
// fill the third place (measured, 64 / 32 keys, us: 6 sequences, 500 queries,
// about 10,000 keys, 16 / 4 heads 450 / 398; 4, 1500, 6000 with a mask
// 328 / 309) and 64 where they don't (10 sequences, 300, about 2000, 8 heads
// 48 / 53) or have few blocks (1000, 128, 128, 8 heads 192 / 197).
//
// What bounds it, measured: many rows, the power limit and the exponentials.
// 8 sequences, 2048 queries, 8192 keys, 16 heads x 128 take 1,060 to 1,080 us,
// 1,020 to 1,040 TFLOP/s, at 1.7 to 1.8 GHz with the MFMA pipe and the VALU half
// busy; 16 x 64 take 615 to 620 us, 890 TFLOP/s, 16 x 32 429, 640, where a score
// costs the VALU the same (78 and 92 % busy) and the MFMAs a half and a quarter.
// Few rows, memory: one query of 32 / 8 heads x 128 over 100,003 keys streams them
// in 74 to 78 us, 5.3 to 5.5 TB/s, and joins in 6.  Small calls, a wave's chain:
// about 0.6 us per block of 32 keys (MFMA and LDS latencies; a deeper ring of
// blocks changes nothing).
//
// Tried and dropped: K a block ahead of V, so that the scores of the next block
// run under the exponentials of this one (48 spilled registers at d_head 128,
// 410 -> 523 us); the sum of the rounded probabilities by dot products (-1 to
// -2 %); four waves per SIMD at d_head 32 (16 spilled, 189 -> 242 us).
#include <float.h>
#include <math.h>

#include <algorithm>

#include "cross.h"
#include "device_common.h"

namespace surge {
namespace {

// LDS rows of CPR 16-byte chunks (DH bf16); chunk c of row r is stored at
// position c ^ f(r), with
//   CPR = 16: f(r) = 4 (r & 3) + (r / 4 & 3),
//   CPR = 8:  f(r) = 4 (r / 2 & 1) + (r / 4 & 3),
//   CPR = 4:  as swz().
// Two reads are served without bank conflicts: K's, one chunk of 32 rows (the
// 16 lanes that the LDS serves together fall on slots of their own, as f takes
// each value for rows of one position), and V's transposing read, whose 32
// lanes take 64 bytes of each of four consecutive rows: bit 2 and up of f put
// them on different 64 bytes.  (With f(r) = r & 15 and swz<8>() the latter
// were conflicts, 59 and 32 % of the LDS's busy cycles.)
template <int CPR>
__device__ __forceinline__ int kv_slot(int row, int chunk) {
  if constexpr (CPR == 16) return row * 16 + (chunk ^ ((row & 3) << 2 | (row >> 2 & 3)));
  if constexpr (CPR == 8) return row * 8 + (chunk ^ ((row >> 1 & 1) << 2 | (row >> 2 & 3)));
  return swz<4>(row, chunk);
}
// The logical chunk of the slot that lane l fills with copy `copy` of a block.
template <int CPR>
__device__ __forceinline__ int kv_copy_chunk(int lane, int copy) {
  if constexpr (CPR == 16) return (lane & 15) ^ ((lane >> 4) << 2 | (copy & 3));
  if constexpr (CPR == 8) return (lane & 7) ^ ((lane >> 4 & 1) << 2 | (copy & 1) << 1 | lane >> 5);
  return copy_chunk<4>(lane, copy);
}

// v combined with its value in lane ^ 32: an exchange in registers, where one
// through LDS would be a latency of it in every block's chain.
template <class Op>
__device__ __forceinline__ float with_other_half(float v, Op op) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return op(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// WAVES waves of 32 rows against blocks of KB keys that they share in LDS, the
// next block copied while the current one is on the MFMA units.
template <int DH, int WAVES, int KB>
__global__ __launch_bounds__(64 * WAVES)
__attribute__((amdgpu_waves_per_eu(DH == 128 && KB == 64 ? 2 : 3))) void cross_kernel(
    CrossAttention a, const CrossItem* items) {
  constexpr int KSTEPS = DH / 16, DT = DH / 32, CPR = DH / 8;
  constexpr int RPC = 64 / CPR;          // rows that a copy instruction fills
  constexpr int NCP = KB / RPC / WAVES;  // copies per wave of a block of K or V
  constexpr int T = KB / 32;             // 32-key tiles of a block
  constexpr uint32_t ROW = DH * 2, BUF = KB * ROW;  // bytes of an LDS row, of a block
  constexpr uint64_t FULL = KB == 64 ? ~0ull : 0xffffffffull;
  static_assert((KB == 32 || KB == 64) && NCP >= 1, "a block is copied by whole instructions");
  __shared__ __attribute__((aligned(256))) u32x4 sKV[4 * BUF / 16];  // K blocks by parity, then V blocks
  __shared__ f32x4 sBias[WAVES][16];  // what a wave adds to its scores: 0 or -inf by key
  const int lane = threadIdx.x & 63, col = lane & 31, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kvh = blockIdx.x % a.n_kv_heads;
  const CrossItem item = items[blockIdx.x / a.n_kv_heads];
  const int G = a.group;
  const int row0 = item.row0 + wave * 32;
  const bool active = row0 < item.rows;  // a wave without rows still copies
  const int row = min(row0 + col, item.rows - 1);
  const int64_t token = (int64_t)item.q_beg + row / G;
  const int head = kvh * G + row % G;

  bf16x8 qf[KSTEPS];
#pragma unroll
  for (int kk = 0; kk < KSTEPS; ++kk)
    qf[kk] = *reinterpret_cast<const bf16x8*>(a.q + token * a.ld_q + head * DH + (kk * 2 + half) * 8);

  const int n_keys = item.k1 - item.k0;
  const int n = (n_keys + KB - 1) / KB;
  const uint16_t* kb = a.k + ((int64_t)item.kv_beg + item.k0) * a.ld_k + kvh * DH;
  const uint16_t* vb = a.v + ((int64_t)item.kv_beg + item.k0) * a.ld_v + kvh * DH;
  const uint8_t* mask = a.mask ? a.mask + item.kv_beg + item.k0 : nullptr;
  const uint32_t lds = lds_address(sKV);
  const uint32_t lcopy = __builtin_amdgcn_readfirstlane(lds + wave * (NCP * 1024));
  // This wave's copies of block i into buffer i % 2; rows past the unit's
  // keys are read clamped.
  auto copy_block = [&](const uint16_t* base, int64_t ld, int i, uint32_t to) {
    const uint16_t* src = base + (int64_t)i * KB * ld;
#pragma unroll
    for (int j = 0; j < NCP; ++j) {
      const int jj = wave * NCP + j;
      const uint32_t r = (uint32_t)min(jj * RPC + lane / CPR, n_keys - 1 - i * KB);
      copy_to_lds16_at(src, r * (uint32_t)ld * 2u + (uint32_t)kv_copy_chunk<CPR>(lane, jj) * 16u,
                       lcopy + to + j * 1024);
    }
  };
  auto copy_kv = [&](int i) {
    copy_block(kb, a.ld_k, i, (i & 1) * BUF);
    copy_block(vb, a.ld_v, i, (2 + (i & 1)) * BUF);
  };
  // The mask's byte of key KB i + lane (% 32 of a 32-key block).
  auto mask_byte = [&](int i) -> uint32_t {
    return mask ? mask[min(i * KB + (lane & (KB - 1)), n_keys - 1)] : 1u;
  };

  // LDS addresses.  K: chunk 2 kk + half of row col; the swizzle is an
  // exclusive or, so step kk is one of the address.  V: 4 features of key 16 c
  // + 8 h + tr_key from dt 32 + tr_feat on; the swizzle of h and dt likewise.
  const int tr_key = 4 * half + ((lane & 15) >> 2);
  const int tr_feat = 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
  uint32_t ka = lds + (uint32_t)kv_slot<CPR>(col, half) * 16u;
  uint32_t va = lds + 2 * BUF + (uint32_t)kv_slot<CPR>(tr_key, tr_feat >> 3) * 16u + (tr_feat & 7) * 2u;
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

  // The maximum starts from the lowest finite value, which scores of -inf don't
  // move: their exponentials are 0 against it, and NaN against themselves.
  bool seen = false;    // any key so far: one for all rows
  bool coarse = false;  // some row's maximum is 2^24 or more
  float m_ref = -FLT_MAX, l_run = 0.0f;
  f32x16 o[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[dt][r] = 0.0f;

  // A block's mask is loaded a block ahead and looked at where it is used: a
  // comparison at once would wait for the copies before it.
  uint32_t byte = 0;
  if (n > 0) {
    copy_kv(0);
    byte = mask_byte(0);
  }
  for (int i = 0; i < n; ++i) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    const bool on = byte != 0 && i * KB + (lane & (KB - 1)) < n_keys;
    const uint64_t keys = __ballot(on) & FULL;
    if (keys != FULL) {
      // Absent keys: -inf in the accumulators that their scores start from, and
      // zeros over what stands in their rows of K and V, where a NaN or an
      // infinity would reach the products.
      reinterpret_cast<float*>(sBias[wave])[lane] = on ? 0.0f : -INFINITY;
      const uint32_t own = (uint32_t)(keys >> (wave * NCP * RPC));  // of the rows that this wave copied
      u32x4* const k_rows = sKV + (i & 1) * (BUF / 16) + wave * (NCP * 64) + lane;
#pragma unroll
      for (int j = 0; j < NCP; ++j)
        if (!(own >> (j * RPC + lane / CPR) & 1u)) {
          k_rows[j * 64] = u32x4{0u, 0u, 0u, 0u};
          k_rows[2 * (BUF / 16) + j * 64] = u32x4{0u, 0u, 0u, 0u};
        }
    }
    __syncthreads();  // the block is there, the other one read out
    if (i + 1 < n) {
      copy_kv(i + 1);
      byte = mask_byte(i + 1);
    }
    if (active && keys) {
      seen = true;
      f32x16 s[T];
      // Ahead of the waves of the SIMD that are at their exponentials.
      __builtin_amdgcn_s_setprio(1);
      auto step = [&](int t, int kk, const f32x16& c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(k_fragment(t, kk), qf[kk], c, 0, 0, 0);
      };
      // (Two ways to the first step, so that the one without absent keys starts
      // from the constant 0.)
      if (keys == FULL) {
        f32x16 zero;
#pragma unroll
        for (int r = 0; r < 16; ++r) zero[r] = 0.0f;
#pragma unroll
        for (int t = 0; t < T; ++t) s[t] = step(t, 0, zero);
      } else {
#pragma unroll
        for (int t = 0; t < T; ++t) {
          f32x16 bias;
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            const f32x4 v = sBias[wave][t * 8 + 2 * g + half];
#pragma unroll
            for (int r = 0; r < 4; ++r) bias[4 * g + r] = v[r];
          }
          s[t] = step(t, 0, bias);
        }
      }
#pragma unroll
      for (int kk = 1; kk < KSTEPS; ++kk)
#pragma unroll
        for (int t = 0; t < T; ++t) s[t] = step(t, kk, s[t]);
      __builtin_amdgcn_s_setprio(0);
      float mloc = s[0][0];
#pragma unroll
      for (int r = 1; r < 16 * T; ++r) mloc = fmaxf(mloc, s[r >> 4][r & 15]);
      mloc = with_other_half(mloc, [](float x, float y) { return fmaxf(x, y); }) * a.scale_log2;
      // The reference of the exponentials follows the maximum only where that
      // has grown by more than 2^8: the probabilities stay below 2^8.
      if (__any(mloc > m_ref + 8.0f)) {
        const float m_new = fmaxf(m_ref, mloc);
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
      // exponentials by up to half of its step: a factor common to all of them
      // while that is small, zeros or infinities where it is not.  There the
      // products are rounded too (looked at where the reference changes, within 1 %
      // of the time without; at every block 1 to 3 %).
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
  l_run = with_other_half(l_run, [](float x, float y) { return x + y; });

  // Register r of tile dt: feature dt 32 + 8 (r / 4) + 4 half + r % 4 of row col.
  if (item.part < 0) {
    // Staged in LDS, so that whole rows are stored (8 bytes a lane from the
    // registers are four times as many requests).
    __syncthreads();  // every wave has read its last block
    if (!active) return;
    // A sum of 0 over some keys (scores that overflow) is no row without keys.
    const float inv = seen ? 1.0f / l_run : 0.0f;
    u32x4* stage = sKV + wave * (32 * CPR);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        uint2 w;
        w.x = pack_bf16x2(o[dt][4 * g] * inv, o[dt][4 * g + 1] * inv);
        w.y = pack_bf16x2(o[dt][4 * g + 2] * inv, o[dt][4 * g + 3] * inv);
        reinterpret_cast<uint2*>(stage + kv_slot<CPR>(col, dt * 4 + g))[half] = w;
      }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
    for (int j = 0; j < CPR / 2; ++j) {
      const int r = row0 + j * RPC + lane / CPR;
      const u32x4 w = stage[j * 64 + lane];
      if (r < item.rows) {
        uint16_t* to = a.out + ((int64_t)item.q_beg + r / G) * a.ld_out + (kvh * G + r % G) * DH;
        __builtin_nontemporal_store(w, reinterpret_cast<u32x4*>(to + kv_copy_chunk<CPR>(lane, j) * 8));
      }
    }
    return;
  }
  if (row0 + col >= item.rows) return;
  const int64_t slot = ((int64_t)(item.part + wave) * a.n_kv_heads + kvh) * 32 + col;
  // -inf is the maximum of a part without keys alone: one of NaN scores, which
  // leave the maximum where it was, has a NaN sum and output to be joined.
  if (half == 0) a.part_ml[slot] = make_float2(seen ? m_ref : -INFINITY, l_run);
  float* po = a.part_o + slot * DH;
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int g = 0; g < 4; ++g)
      *reinterpret_cast<float4*>(po + dt * 32 + g * 8 + half * 4) =
          make_float4(o[dt][4 * g], o[dt][4 * g + 1], o[dt][4 * g + 2], o[dt][4 * g + 3]);
}

// Joins the parts of a row of one key head in WAVES waves: wave w takes parts
// w, w + WAVES, ..., BATCH loads in flight, and the waves are added in order.
// A workgroup has ROWS rows.
template <int DH, int WAVES, int ROWS, int BATCH>
__global__ __launch_bounds__(64 * WAVES * ROWS) void cross_join_kernel(CrossAttention a) {
  constexpr int PER = DH < 64 ? 1 : DH / 64;
  static_assert(WAVES == 1 || ROWS == 1, "waves that meet have one row");
  __shared__ float sm[WAVES], so[WAVES][DH + 1];
  const int lane = threadIdx.x & 63;
  const int wave = WAVES == 1 ? 0 : threadIdx.x >> 6;
  const int first = blockIdx.x / a.n_kv_heads * ROWS;
  const int kvh = blockIdx.x % a.n_kv_heads;
  const CrossJoin j = a.joins[first / 32];
  const int r = first % 32 + (WAVES == 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0);
  if (r >= j.rows) return;
  auto slot = [&](int p) {
    return ((int64_t)(j.part0 + p * j.stride) * a.n_kv_heads + kvh) * 32 + r;
  };
  float m = -INFINITY;
  for (int p = wave * 64 + lane; p < j.parts; p += 64 * WAVES) m = fmaxf(m, a.part_ml[slot(p)].x);
  m = wave_max(m);
  if constexpr (WAVES > 1) {
    if (lane == 0) sm[wave] = m;
    __syncthreads();
    m = sm[0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) m = fmaxf(m, sm[w]);
  }
  float l = 0.0f, o[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) o[i] = 0.0f;
  // Without any key for the row (m = -inf) every part is zeros: nothing to add.
  for (int p0 = wave; p0 < j.parts && m > -INFINITY; p0 += WAVES * BATCH) {
    float2 ml[BATCH];
    float v[BATCH][PER];
#pragma unroll
    for (int q = 0; q < BATCH; ++q) {
      const int64_t s = slot(min(p0 + q * WAVES, j.parts - 1));
      ml[q] = a.part_ml[s];
#pragma unroll
      for (int i = 0; i < PER; ++i) v[q][i] = lane < DH ? a.part_o[s * DH + lane * PER + i] : 0.0f;
    }
#pragma unroll
    for (int q = 0; q < BATCH; ++q) {
      const float f = p0 + q * WAVES < j.parts ? __builtin_amdgcn_exp2f(ml[q].x - m) : 0.0f;
      l = fmaf(f, ml[q].y, l);
#pragma unroll
      for (int i = 0; i < PER; ++i) o[i] = fmaf(f, v[q][i], o[i]);
    }
  }
  if constexpr (WAVES > 1) {
    if (lane == 0) so[wave][DH] = l;
    if (lane < DH)
#pragma unroll
      for (int i = 0; i < PER; ++i) so[wave][lane * PER + i] = o[i];
    __syncthreads();
    if (wave > 0) return;
#pragma unroll
    for (int w = 1; w < WAVES; ++w) {
      l += so[w][DH];
#pragma unroll
      for (int i = 0; i < PER; ++i)
        if (lane < DH) o[i] += so[w][lane * PER + i];
    }
  }
  const float inv = m > -INFINITY ? 1.0f / l : 0.0f;
  const int row = j.row0 + r;
  uint16_t* out = a.out + ((int64_t)j.q_beg + row / a.group) * a.ld_out + (kvh * a.group + row % a.group) * DH;
  if constexpr (PER == 2)
    reinterpret_cast<uint32_t*>(out)[lane] = pack_bf16x2(o[0] * inv, o[1] * inv);
  else if (lane < DH)
    out[lane] = (uint16_t)(pack_bf16x2(o[0] * inv, 0.0f) & 0xffffu);
}

template <int DH>
hipError_t launch(const CrossAttention& a, hipStream_t stream) {
  const unsigned h = (unsigned)a.n_kv_heads;
  const CrossItem* items = a.items;
#define SURGE_LAUNCH(CLASS, WAVES, KB)                                                               \
  hipLaunchKernelGGL((cross_kernel<DH, WAVES, KB>), dim3(a.n_items[CLASS] * h), dim3(64 * WAVES), 0, \
                     stream, a, items)
  constexpr int SHORT = DH == 128 ? 32 : 64;  // the plan takes short blocks for DH 128 alone
  if (a.n_items[0] > 0 && a.short_blocks) SURGE_LAUNCH(0, 4, SHORT);
  if (a.n_items[0] > 0 && !a.short_blocks) SURGE_LAUNCH(0, 4, 64);
  items += a.n_items[0];
  if (a.n_items[1] > 0) SURGE_LAUNCH(1, 2, 32);
  items += a.n_items[1];
  if (a.n_items[2] > 0) SURGE_LAUNCH(2, 1, 32);
#undef SURGE_LAUNCH
  const unsigned rows = (unsigned)a.n_joins * 32;
  if (a.n_joins > 0 && a.max_parts > 64)
    hipLaunchKernelGGL((cross_join_kernel<DH, 16, 1, 8>), dim3(rows * h), dim3(1024), 0, stream, a);
  else if (a.n_joins > 0 && a.max_parts > 8)
    hipLaunchKernelGGL((cross_join_kernel<DH, 4, 1, 8>), dim3(rows * h), dim3(256), 0, stream, a);
  else if (a.n_joins > 0)
    hipLaunchKernelGGL((cross_join_kernel<DH, 1, 4, 4>), dim3(rows / 4 * h), dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_cross_attention(const CrossAttention& a, int d_head, hipStream_t stream) {
  if (d_head == 32) return launch<32>(a, stream);
  if (d_head == 64) return launch<64>(a, stream);
  return launch<128>(a, stream);
}

}  // namespace surge
