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
// A unit is 32 rows of one (sequence, key head) over a range of its keys.  A
// wave computes S^T = K Q^T with 32x32x16 MFMAs, so that a lane owns one row
// (running maximum, sum and rescaling are the lane's own, joined with lane ^
// 32 that has the other half of a key block), keeps the probabilities in
// registers as the operand of O^T += V^T P^T, and reads V^T from the
// row-major V block with the transposing LDS read.  Where one (sequence, key
// head)'s keys are split over units, each writes its maximum, sum and
// unnormalised output in fp32, and a second kernel joins them in key order.
#include <math.h>

#include <algorithm>

#include "cross.h"
#include "device_common.h"

namespace surge {
namespace {

// Chunk c of LDS row r (DH bf16) is stored at c ^ f(r): as swz() for rows of
// 4 or 8 chunks, r & 15 for 16, so that the 16 lanes that the LDS serves
// together in a read of one chunk from 32 rows fall on slots of their own.
template <int CPR>
__device__ __forceinline__ int kv_slot(int row, int chunk) {
  if constexpr (CPR == 16)
    return row * 16 + (chunk ^ (row & 15));
  else
    return swz<CPR>(row, chunk);
}
template <int CPR>
__device__ __forceinline__ int kv_copy_chunk(int lane, int copy) {
  if constexpr (CPR == 16)
    return (lane & 15) ^ ((4 * copy + (lane >> 4)) & 15);
  else
    return copy_chunk<CPR>(lane, copy);
}

template <int DH>
__global__ __launch_bounds__(64) void cross_attention_kernel(CrossAttention a) {
  constexpr int KSTEPS = DH / 16, DT = DH / 32, CPR = DH / 8;
  constexpr int RPC = 64 / CPR, NCP = 32 / RPC, BLK = 32 * CPR;
  __shared__ u32x4 sK[2][BLK];
  __shared__ u32x4 sV[2][BLK];
  const int lane = threadIdx.x, col = lane & 31, half = lane >> 5;
  const int kvh = blockIdx.x % a.n_kv_heads;
  const CrossItem item = a.items[blockIdx.x / a.n_kv_heads];
  const int G = a.group;
  const int row = min(item.row0 + col, item.rows - 1);
  const int64_t token = (int64_t)item.q_beg + row / G;
  const int head = kvh * G + row % G;

  bf16x8 qf[KSTEPS];
#pragma unroll
  for (int kk = 0; kk < KSTEPS; ++kk)
    qf[kk] = *reinterpret_cast<const bf16x8*>(a.q + token * a.ld_q + head * DH + (kk * 2 + half) * 8);

  const uint16_t* kb = a.k + (int64_t)item.kv_beg * a.ld_k + kvh * DH;
  const uint16_t* vb = a.v + (int64_t)item.kv_beg * a.ld_v + kvh * DH;
  const uint8_t* mask = a.mask ? a.mask + item.kv_beg : nullptr;
  const uint32_t lk = lds_address(sK[0]), lv = lds_address(sV[0]);
  auto copy_block = [&](int k0, int b) {
#pragma unroll
    for (int j = 0; j < NCP; ++j) {
      const int r = min(k0 + j * RPC + lane / CPR, item.k1 - 1);
      const int c = kv_copy_chunk<CPR>(lane, j) * 8;
      copy_to_lds16(kb + r * a.ld_k + c, lk + b * (BLK * 16) + j * 1024);
      copy_to_lds16(vb + r * a.ld_v + c, lv + b * (BLK * 16) + j * 1024);
    }
  };

  float m_run = -INFINITY, l_run = 0.0f;
  f32x16 o[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[dt][r] = 0.0f;
  const int tr_key = 4 * half + ((lane & 15) >> 2);
  const int tr_feat = 16 * ((lane >> 4) & 1) + 4 * (lane & 3);

  int b = 0;
  if (item.k0 < item.k1) copy_block(item.k0, 0);
  for (int k0 = item.k0; k0 < item.k1; k0 += 32, b ^= 1) {
    // Key k0 + col is there and not masked, as bit col of `keys`.
    const int kc = k0 + col;
    bool on = kc < item.k1;
    if (mask && on) on = mask[kc] != 0;
    const uint32_t keys = (uint32_t)__ballot(on);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    if (k0 + 32 < item.k1) copy_block(k0 + 32, b ^ 1);
    if (keys == 0) continue;
    if (keys != ~0u) {
      // What stands in the V rows of absent keys must not reach the products,
      // where a NaN or infinity times 0 would.
#pragma unroll
      for (int j = 0; j < NCP; ++j)
        if (!(keys >> (j * RPC + lane / CPR) & 1)) sV[b][j * 64 + lane] = u32x4{0u, 0u, 0u, 0u};
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
    f32x16 s;
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = 0.0f;
#pragma unroll
    for (int kk = 0; kk < KSTEPS; ++kk)
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
          __builtin_bit_cast(bf16x8, sK[b][kv_slot<CPR>(col, kk * 2 + half)]), qf[kk], s, 0, 0, 0);
    if (keys != ~0u) {
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (!(keys >> (8 * (r >> 2) + 4 * half + (r & 3)) & 1)) s[r] = -INFINITY;
    }
    float mloc = s[0];
#pragma unroll
    for (int r = 1; r < 16; ++r) mloc = fmaxf(mloc, s[r]);
    mloc = fmaxf(mloc, __shfl_xor(mloc, 32, 64));
    const float m_new = fmaxf(m_run, mloc * a.scale_log2);
    float psum = 0.0f;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], a.scale_log2, -m_new));
      psum += s[r];
    }
    psum += __shfl_xor(psum, 32, 64);
    const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);
    l_run = fmaf(l_run, alpha, psum);
    m_run = m_new;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[dt][r] *= alpha;
    bf16x8 pb[2];
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
      for (int j = 0; j < 8; ++j) pb[c][j] = (__bf16)s[8 * c + j];
    const char* vbytes = reinterpret_cast<const char*>(sV[b]);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      const int feat = dt * 32 + tr_feat;
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        bf16x4 v2[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const char* pa = vbytes + kv_slot<CPR>(16 * c + 8 * i + tr_key, feat >> 3) * 16 + (feat & 7) * 2;
          v2[i] = __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                                 (__attribute__((address_space(3))) i16x4*)pa));
        }
        const bf16x8 va = __builtin_shufflevector(v2[0], v2[1], 0, 1, 2, 3, 4, 5, 6, 7);
        o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va, pb[c], o[dt], 0, 0, 0);
      }
    }
  }

  // Register r of tile dt: feature dt 32 + 8 (r / 4) + 4 half + r % 4.
  if (item.row0 + col >= item.rows) return;
  if (item.part < 0) {
    const float inv = l_run > 0.0f ? 1.0f / l_run : 0.0f;
    uint16_t* out = a.out + token * a.ld_out + head * DH;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        uint2 w;
        w.x = pack_bf16x2(o[dt][4 * g] * inv, o[dt][4 * g + 1] * inv);
        w.y = pack_bf16x2(o[dt][4 * g + 2] * inv, o[dt][4 * g + 3] * inv);
        *reinterpret_cast<uint2*>(out + dt * 32 + g * 8 + half * 4) = w;
      }
    return;
  }
  const int64_t slot = ((int64_t)item.part * a.n_kv_heads + kvh) * 32 + col;
  if (half == 0) a.part_ml[slot] = make_float2(m_run, l_run);
  float* po = a.part_o + slot * DH;
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int g = 0; g < 4; ++g)
      *reinterpret_cast<float4*>(po + dt * 32 + g * 8 + half * 4) =
          make_float4(o[dt][4 * g], o[dt][4 * g + 1], o[dt][4 * g + 2], o[dt][4 * g + 3]);
}

// Joins the parts of one row: a wave per (row, key head), in key order.
template <int DH>
__global__ __launch_bounds__(64) void cross_join_kernel(CrossAttention a) {
  const int kvh = blockIdx.x % a.n_kv_heads;
  const int unit = blockIdx.x / a.n_kv_heads;
  const CrossJoin j = a.joins[unit / 32];
  const int r = unit % 32;
  if (r >= j.rows) return;
  const int lane = threadIdx.x;
  float m = -INFINITY;
  for (int p = 0; p < j.parts; ++p)
    m = fmaxf(m, a.part_ml[((int64_t)(j.part0 + p) * a.n_kv_heads + kvh) * 32 + r].x);
  constexpr int PER = DH < 64 ? 1 : DH / 64;
  float l = 0.0f, o[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) o[i] = 0.0f;
  if (m > -INFINITY)
    for (int p = 0; p < j.parts; ++p) {
      const int64_t slot = ((int64_t)(j.part0 + p) * a.n_kv_heads + kvh) * 32 + r;
      const float2 ml = a.part_ml[slot];
      const float f = __builtin_amdgcn_exp2f(ml.x - m);
      l = fmaf(f, ml.y, l);
#pragma unroll
      for (int i = 0; i < PER; ++i)
        if (lane + 64 * i < DH) o[i] = fmaf(f, a.part_o[slot * DH + lane + 64 * i], o[i]);
    }
  const float inv = l > 0.0f ? 1.0f / l : 0.0f;
  const int row = j.row0 + r;
  uint16_t* out = a.out + ((int64_t)j.q_beg + row / a.group) * a.ld_out + (kvh * a.group + row % a.group) * DH;
#pragma unroll
  for (int i = 0; i < PER; ++i)
    if (lane + 64 * i < DH) out[lane + 64 * i] = (uint16_t)(pack_bf16x2(o[i] * inv, 0.0f) & 0xffffu);
}

}  // namespace

hipError_t launch_cross_attention(const CrossAttention& a, int d_head, int n_items, int n_joins,
                                  hipStream_t stream) {
  if (n_items <= 0) return hipSuccess;
  const dim3 grid((unsigned)((int64_t)n_items * a.n_kv_heads));
  const dim3 join((unsigned)((int64_t)n_joins * 32 * a.n_kv_heads));
#define SURGE_LAUNCH(DH)                                                                     \
  do {                                                                                       \
    hipLaunchKernelGGL((cross_attention_kernel<DH>), grid, dim3(64), 0, stream, a);          \
    if (n_joins > 0) hipLaunchKernelGGL((cross_join_kernel<DH>), join, dim3(64), 0, stream, a); \
  } while (0)
  if (d_head == 32)
    SURGE_LAUNCH(32);
  else if (d_head == 64)
    SURGE_LAUNCH(64);
  else
    SURGE_LAUNCH(128);
#undef SURGE_LAUNCH
  return hipGetLastError();
}

}  // namespace surge
