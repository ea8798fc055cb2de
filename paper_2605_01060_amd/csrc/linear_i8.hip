// Linear layers in 8-bit integers (gfx950): y = epi(sx[m] sw[n] (X W^T)[m][n]
// + b[n]), X [M, K] int8 with a scale per token, W [N, K] int8 with a scale
// per output channel.  The products are summed exactly in 32-bit integers
// (K <= 65,536 of at most 2^14 each), so only the finish rounds: one
// conversion to fp32, two products, the bias, GELU or residual, and bf16.
//
// A row's 128 bytes of a K stage are laid out as the bf16 layers lay out
// their 64 values: a fragment of a 16x16x64 MFMA is 16 rows x four 16-byte
// chunks, read from LDS rows whose chunk c of row r sits at c ^ (r & 7).
//
// Three kinds of kernel, chosen by a model of their times (below): persistent
// 256 x 256 and 192 x 256 tiles with the schedule of linear_wide.hip (its waits
// and barriers stand there a second time: a mend of one is one of both), rings of
// one tile per workgroup for launches of few tiles, and a kernel for few
// tokens.
//
// What bounds them, measured: large K, the power limit (8192^3 in 380 us where
// the card is cool, 2,892 TOP/s, in 449 many times in a row, 2,450; M = 200,003, N =
// 1024, K = 4096 with residual 730 to 820 us, 2,050 to 2,300); K = 768, the
// epilogue, during which a CU's MFMA pipe idles (M = 200,003, N = 2304: 370 to 430
// us, 1,650 to 1,910 TOP/s at 1.9 GHz, MFMA pipe 49 % busy, VALU 41 %); few tiles, a
// tile's chain of K stages (0.26 us each); one token, 2.9 us, the latencies of a
// launch, two loads and a meeting of eight waves.
//
// Tried and dropped: starting the CUs apart, so that their stores do not come
// at once (it costs its delay and gains nothing); the channel vectors in
// registers over the epilogue's passes (+-1 %); two workgroups of 128 x 256
// tiles on a CU, one's epilogue under the other's MFMAs (M = 200,003, N = 2304, K =
// 768 406 -> 487 us: two thirds of the MFMAs per copied byte);
// ordinary instead of nontemporal output stores (400 -> 416 us).
#include <algorithm>

#include "linear_common.h"
#include "reader.h"

namespace surge {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));

// Four consecutive channels of one token.
template <int EPI>
__device__ __forceinline__ uint2 finish_i8(i32x4 v, float sx, float4 sw, float4 bb, uint2 res) {
  const float s[4] = {(float)v[0] * sx * sw.x, (float)v[1] * sx * sw.y, (float)v[2] * sx * sw.z,
                      (float)v[3] * sx * sw.w};
  return finish4<EPI>(s, bb, bb, bb, bb, 0.0f, 0.0f, res);
}

__device__ __forceinline__ i32x4 lds_fragment(uint32_t addr) {
  return __builtin_bit_cast(i32x4, *(const __attribute__((address_space(3))) u32x4*)addr);
}
__device__ __forceinline__ i32x4 mma(i32x4 w, i32x4 x, i32x4 c) {
  return __builtin_amdgcn_mfma_i32_16x16x64_i8(w, x, c, 0, 0, 0);
}

// A wave's part of a tile's epilogue, as store_tile of the bf16 layers: passes
// of 32 tokens x 64 channels over a region of its own in LDS, residual rows
// loaded ahead, whole 128-byte row segments stored.  slot16(r, c): 16-byte
// slot c of region row r.  vec(v, q): the scales (v = 0) or biases (1) of the
// wave's channels 4 q .. 4 q + 3.  scale(r): the scale of the wave's row r.
template <int TJ, int TI, int EPI, class Slot, class Vec, class Scale>
__device__ __forceinline__ void store_i8(const i32x4 (&acc)[TI][TJ], Slot slot16, Vec vec, Scale scale,
                                         const LinearI8& a, int mw, int nw, int M, int N, int lane) {
  constexpr bool RES = EPI == EPI_BIAS_RESIDUAL;
  constexpr int PI = TI / 4;         // 64-channel groups
  constexpr int NP = (TJ / 2) * PI;  // passes
  static_assert(TI % 4 == 0 && TJ % 2 == 0, "epilogue passes are 32 rows x 64 channels");
  const int l16 = lane & 15, lq = lane >> 4;
  const int cr = lane >> 3;  // row within the 8 rows of one coalesced access
  const int cp = lane & 7;   // 16-byte pair within a row
  u32x4 rv[RES ? NP : 1][4];
  if constexpr (RES) {
#pragma unroll
    for (int p = 0; p < NP; ++p)
#pragma unroll
      for (int it = 0; it < 4; ++it) {
        const int m = min(mw + p / PI * 32 + it * 8 + cr, M - 1);
        const int n = min(nw + p % PI * 64 + 8 * cp, N - 8);
        rv[p][it] = __builtin_nontemporal_load(
            reinterpret_cast<const u32x4*>(a.res + (int64_t)m * a.ld_res + n));
      }
  }
#pragma unroll
  for (int p = 0; p < NP; ++p) {
    const int j = p / PI, ip = p % PI;
    if constexpr (RES) {
#pragma unroll
      for (int it = 0; it < 4; ++it) {
        const int r = it * 8 + cr;
        const int ph = (2 * cp) ^ rsw(r);  // physical unit of logical unit 2 cp
        u32x4 v = rv[p][it];
        if (ph & 1) v = u32x4{v[2], v[3], v[0], v[1]};
        *slot16(r, ph >> 1) = v;
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
    float sx[2];
#pragma unroll
    for (int jj = 0; jj < 2; ++jj) sx[jj] = scale(j * 32 + jj * 16 + l16);
#pragma unroll
    for (int ii = 0; ii < 4; ++ii) {
      const float4 sw = vec(0, 4 * (4 * ip + ii) + lq), bb = vec(1, 4 * (4 * ip + ii) + lq);
#pragma unroll
      for (int jj = 0; jj < 2; ++jj) {
        const int r = jj * 16 + l16;
        uint2& cell = reinterpret_cast<uint2*>(slot16(r, 0))[(4 * ii + lq) ^ rsw(r)];
        cell = finish_i8<EPI>(acc[4 * ip + ii][2 * j + jj], sx[jj], sw, bb, RES ? cell : uint2{0u, 0u});
      }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // region written by all lanes
    u32x4 ov[4];
#pragma unroll
    for (int it = 0; it < 4; ++it) {
      const int r = it * 8 + cr;
      const int ph = (2 * cp) ^ rsw(r);
      ov[it] = *slot16(r, ph >> 1);
      if (ph & 1) ov[it] = u32x4{ov[it][2], ov[it][3], ov[it][0], ov[it][1]};
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // region free for the next pass
    // Everything issued before the tile's first store is done by here: the
    // copies in flight retire before the stores and need not wait for them.
    if (p == 0) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
    for (int it = 0; it < 4; ++it) {
      const int m = mw + j * 32 + it * 8 + cr, n = nw + ip * 64 + 8 * cp;
      if (m < M && n < N)
        __builtin_nontemporal_store(ov[it], reinterpret_cast<u32x4*>(a.y + (int64_t)m * a.ld_y + n));
    }
  }
}

// WAVES_M x WAVES_N waves of 16 (J0 + J1) tokens x 16 TI features; phase 0
// takes J0 of a wave's token fragments, phase 1 the other J1.
template <int WAVES_M, int WAVES_N, int TI, int J0, int J1, int EPI>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2))) void linear_i8_wide_kernel(
    LinearI8 a, int M, int K, int tiles_n, int n_tiles) {
  constexpr int TJ = J0 + J1;
  constexpr int R0 = 16 * J0, R1 = 16 * J1;  // a wave's token rows of either phase
  constexpr int BM = WAVES_M * (R0 + R1), BN = 256;
  constexpr int C1 = WAVES_M * R1 / 64;      // copies per wave of the phase-1 rows
  constexpr int CPS = 6 + C1;                // ... of a stage: 4 W, 2 phase-0 rows, C1
  static_assert(WAVES_M * WAVES_N == 8 && WAVES_N * TI == 16 && WAVES_M * R0 == 128 &&
                    WAVES_M * R1 == 64 * C1 && C1 <= 2 && J1 == 2 && TI * J0 == 16,
                "tiles of this kernel");
  // LDS, in bytes from smem: a stage of parity p at p * BUF, its W rows, then
  // (X0 on) its phase-0 and (X1 on) phase-1 rows of X, wave_m by wave_m; the
  // spare parts of the epilogue regions, 32 rows less the 8 C1 in copy slots.
  constexpr uint32_t X0 = 32768, X1 = X0 + 16384, BUF = X1 + C1 * 8192, SPARE = 2 * BUF;
  constexpr int SPARE_ROWS = 32 - 8 * C1;
  __shared__ __attribute__((aligned(128))) u32x4 smem[SPARE / 16 + 8 * SPARE_ROWS * 8];
  // The channels' scales and biases and the tokens' scales, by tile parity.
  __shared__ float4 svec[2][2][BN / 4];
  __shared__ float srow[2][256];

  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wave_m = wave / WAVES_N;
  const int wn0 = (wave % WAVES_N) * (16 * TI);
  const int wm0 = wave_m * (R0 + R1);
  const int nkt = K / 128;
  const int G = gridDim.x;

  // Fragment addresses: row lane % 16, then the swizzled 16-byte chunk of the
  // 32-wide K step ks, which for ks = 1 differs in bit 6 of the address only
  // (rows are 128 bytes, aligned); fragments are 16 rows apart.
  const uint32_t lds = lds_address(smem);
  uint32_t aw, ax, ax1;
  i32x4 fw[TI][2], f0[J0][2], f1[J1][2];
  auto read_w = [&](int i, int ks) { fw[i][ks] = lds_fragment((aw ^ ks * 64) + i * 2048); };
  auto read_x0 = [&](int j, int ks) { f0[j][ks] = lds_fragment((ax ^ ks * 64) + j * 2048); };
  auto read_x1 = [&](int j, int ks) {  // (J0 == J1: the same rows, X1 - X0 on)
    f1[j][ks] = lds_fragment(((J0 == J1 ? ax + (X1 - X0) : ax1) ^ ks * 64) + j * 2048);
  };

  // Copies.  A wave instruction fills 8 rows of 128 bytes.
  const uint32_t ldsw = __builtin_amdgcn_readfirstlane(lds + wave * 1024);
  int it_tile = blockIdx.x;  // the copy stream's tile and stage
  int it_kt = 0;
  const int8_t* xs;
  const int8_t* ws;
  uint32_t xo[2 + C1];
  uint32_t wo;
  // A copy of the lane index that the compiler cannot see through: what is
  // derived from it is computed where it is used and not kept in registers
  // over the main loop, which has none to spare.
  auto opaque_lane = [&]() {
    int l = lane;
    asm volatile("" : "+v"(l));
    return l;
  };
  // The addresses that stay the same over a tile but for the stage parity p;
  // formed at its start so that they take no registers over the epilogue.
  // With one register too many the allocator spilled wo, and the compiler
  // then waited for every copy in flight where it was used again, in each
  // K stage.
  auto tile_addresses = [&](uint32_t p) {
    const int l = opaque_lane();
    const uint32_t ch = (uint32_t)swz16(l & 15, l >> 4) * 16u + p * BUF;
    aw = lds + (uint32_t)wn0 * 128u + ch;
    ax = lds + X0 + (uint32_t)(wave_m * R0) * 128u + ch;
    ax1 = lds + X1 + (uint32_t)(wave_m * R1) * 128u + ch;
    wo = __umul24((uint32_t)(wave * 8 + (l >> 3)), (uint32_t)K) +
         (uint32_t)copy_chunk16(l) * 16u;
  };
  auto point = [&]() {
    int tm_, tn_;
    tile_coords<ORDER_ROW_GROUPS>(it_tile, n_tiles, tiles_n, &tm_, &tn_);
    xs = a.x + (int64_t)(tm_ * BM) * a.ld_x;
    ws = a.w + (int64_t)(tn_ * BN) * K;
    const int l = opaque_lane();
#pragma unroll
    for (int q = 0; q < 2 + C1; ++q) {  // copies 0, 1: phase 0; rows past M: clamped
      const int lr = (q & 1) * 64 + wave * 8 + (l >> 3);
      const int row = q < 2 ? lr / R0 * (R0 + R1) + lr % R0 : lr / R1 * (R0 + R1) + R0 + lr % R1;
      xo[q] = __umul24((uint32_t)min(row, M - 1 - tm_ * BM), (uint32_t)a.ld_x) +
              (uint32_t)copy_chunk16(l) * 16u;
    }
  };
  // Copy c of the cursor's stage into parity p, skipped where `go` is 0:
  // 0 .. 3 W, 4 .. 5 the phase-0 rows, 6 on the phase-1 rows.
  auto copy = [&](int c, uint32_t p, uint32_t go) {
    const uint32_t base = ldsw + p * BUF;
    if (c < 4)
      copy_to_lds16_if(ws + (size_t)(c * 64) * K + it_kt * 128, wo, base + c * 8192, go);
    else
      copy_to_lds16_if(xs + it_kt * 128, xo[c - 4], base + X0 + (c - 4) * 8192, go);
  };
  auto advance = [&]() {
    if (++it_kt == nkt) {
      it_kt = 0;
      it_tile += G;
      if (it_tile < n_tiles) point();
    }
  };
  auto more = [&]() { return lane_mask(it_tile < n_tiles); };

  int t = blockIdx.x;  // < n_tiles: the grid is never larger than the tile count
  point();
  tile_addresses(0);
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    const uint32_t go = more();
#pragma unroll
    for (int c = 0; c < CPS; ++c) copy(c, s, go);
    if (s == 0 || go) advance();
  }
  if (more())
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(CPS) : "memory");
  else
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();

  uint32_t p = 0;  // parity of the stage being computed
  int tpar = 0;
  bool first = true;

  for (;;) {
    int tm, tn;
    tile_coords<ORDER_ROW_GROUPS>(t, n_tiles, tiles_n, &tm, &tn);
    const int m0 = tm * BM;
    const int n0 = tn * BN;
    tile_addresses(p);

    // The channels' vectors by waves 0 and 1 and the tokens' scales, 64 a
    // wave, by waves 2 on; published by the barriers of the tile's first
    // stages, last read two tiles ago.
    if (wave < 2) {
      copy_lanes_to_lds16((wave ? a.bias : a.w_scale) + n0, lds_address(&svec[tpar][wave][0]));
    } else if (wave < 2 + BM / 64) {
      const int l = opaque_lane();
      copy_to_lds4_at(a.x_scale + m0, (uint32_t)min((wave - 2) * 64 + l, M - 1 - m0) * 4u,
                      lds_address(&srow[tpar][(wave - 2) * 64]));
    }

    i32x4 acc[TI][TJ];
#pragma unroll
    for (int i = 0; i < TI; ++i)
#pragma unroll
      for (int j = 0; j < TJ; ++j) acc[i][j] = i32x4{0, 0, 0, 0};

    // The tile's first stage: its W and phase-0 rows landed before the last
    // barrier A.
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
#pragma unroll
      for (int j = 0; j < J0; ++j) read_x0(j, ks);
#pragma unroll
      for (int i = 0; i < TI; ++i) read_w(i, ks);
    }

    for (int kt = 0; kt < nkt; ++kt) {
      const bool last = kt == nkt - 1;
      const uint32_t go = more();
      // Phase 0: 16 steps of two MFMAs.
#pragma unroll
      for (int q = 0; q < 16; ++q) {
        const int ks = q >> 3, i = (q & 7) * 2 / J0, j = (q & 7) * 2 % J0;
        acc[i][j] = mma(fw[i][ks], f0[j][ks], acc[i][j]);
        acc[i][j + 1] = mma(fw[i][ks], f0[j + 1][ks], acc[i][j + 1]);
        if (q == 3) {
          // Barrier B: the phase-1 rows of this stage have landed (at a
          // tile's first stage they had before the previous epilogue's first
          // store); W and the phase-0 rows are read out.  CPS copies, or
          // more, were issued after those waited for, unless the stream has
          // ended.
          if (kt > 0) {
            if (go)
              asm volatile("s_waitcnt vmcnt(%0)" ::"n"(CPS) : "memory");
            else
              asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
          }
          __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
          __syncthreads();
        }
        if (q >= 4 && q < 8) read_x1(q & 1, (q - 4) >> 1);
        if (q >= 5 && (q & 1)) copy((q - 5) >> 1, p, go);
        __builtin_amdgcn_sched_barrier(0);
      }
      // Barrier A: W and the phase-0 rows of the next stage have landed (at a
      // tile's first stage as above); the phase-1 rows are read out.  (A tile
      // of one stage publishes its per-feature vectors here.)
      if (kt > 0 || first || nkt == 1) {
        if (go && nkt > 1)
          asm volatile("s_waitcnt vmcnt(%0)" ::"n"(CPS) : "memory");
        else
          asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      }
      __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
      __syncthreads();
      // The next stage is read from the other parity.
      const uint32_t other = p ? 0u - BUF : BUF;
      aw += other;
      ax += other;
      ax1 += other;
      const uint32_t go1 = lane_mask(go && !last);
      __builtin_amdgcn_sched_barrier(0);
      // Phase 1 (the fragments read at a tile's last stage are not used):
      // 2 TI steps of two MFMAs; the 2 J0 phase-0 fragments of the next stage
      // over the last steps.
#pragma unroll
      for (int q = 0; q < 2 * TI; ++q) {
        const int ks = q / TI, i = q % TI;
        acc[i][J0] = mma(fw[i][ks], f1[0][ks], acc[i][J0]);
        acc[i][J0 + 1] = mma(fw[i][ks], f1[1][ks], acc[i][J0 + 1]);
        read_w(i, ks);
        if (i >= TI - J0) read_x0(i - (TI - J0), ks);
        if ((q & 1) && q / 2 < C1) copy(6 + q / 2, p, go1);
        __builtin_amdgcn_sched_barrier(0);
      }
      if (go1) advance();
      p ^= 1;
    }
    first = false;

    // The first region rows beside the stages, the last 8 C1 in this wave's
    // copy slots of the phase-1 rows of the last stage's parity.
    u32x4* const spare = smem + SPARE / 16 + wave * (SPARE_ROWS * 8);
    u32x4* const slots = smem + ((p ^ 1) * BUF + X1) / 16 + wave * 64;
    auto slot16 = [&](int r, int c) -> u32x4* {
      if (r < SPARE_ROWS) return spare + r * 8 + c;
      return slots + (r - SPARE_ROWS >= 8 ? 512 : 0) + (r & 7) * 8 + c;
    };
    auto vec = [&](int v, int q) { return svec[tpar][v][(wn0 >> 2) + q]; };
    auto scale = [&](int r) { return srow[tpar][wm0 + r]; };
    store_i8<TJ, TI, EPI>(acc, slot16, vec, scale, a, m0 + wm0, n0 + wn0, M, INT32_MAX, opaque_lane());

    // The held-back copies, into slots only this wave has used since.
    const uint32_t go = more();
#pragma unroll
    for (int c = 6; c < CPS; ++c) copy(c, p ^ 1, go);
    if (go) advance();
    tpar ^= 1;
    t += G;
    if (t >= n_tiles) break;
  }
}

// Launches of few tiles: WAVES_M x WAVES_N waves of (16 TJ) tokens x 64
// channels, one tile a workgroup, K in 128-byte stages through a ring of
// STAGES LDS buffers: the copies of a stage have STAGES - 1 stages to arrive.
template <int WAVES_M, int WAVES_N, int TJ, int STAGES, int EPI>
__global__ __launch_bounds__(64 * WAVES_M * WAVES_N) __attribute__((amdgpu_waves_per_eu(2))) void
linear_i8_ring_kernel(LinearI8 a, int M, int N, int K, int tiles_n, int n_tiles) {
  constexpr int WAVES = WAVES_M * WAVES_N, TI = 4;
  constexpr int BM = WAVES_M * TJ * 16, BN = WAVES_N * 64;
  constexpr int XC = BM / 8 / WAVES, WC = BN / 8 / WAVES;  // copies per wave of a stage
  constexpr int SLOTS = (BM + BN) * 8;
  static_assert(XC * 8 * WAVES == BM && WC * 8 * WAVES == BN && STAGES * SLOTS >= WAVES * 256,
                "whole copies, and room for the epilogue's regions");
  __shared__ __attribute__((aligned(128))) u32x4 smem[STAGES * SLOTS];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l16 = lane & 15, lq = lane >> 4;
  const int wn0 = wave % WAVES_N * 64, wm0 = wave / WAVES_N * (TJ * 16);
  int tm, tn;
  tile_coords<ORDER_ROW_GROUPS>(blockIdx.x, n_tiles, tiles_n, &tm, &tn);
  const int m0 = tm * BM, n0 = tn * BN;
  const int8_t* xs = a.x + (int64_t)m0 * a.ld_x;
  const int8_t* ws = a.w + (int64_t)n0 * K;
  // Copy j of wave w fills rows (WAVES j + w) 8 .. + 7 of either operand; rows
  // past the matrix are read clamped and never stored.
  uint32_t xo[XC], wo[WC];
#pragma unroll
  for (int j = 0; j < XC; ++j)
    xo[j] = (uint32_t)min((j * WAVES + wave) * 8 + (lane >> 3), M - 1 - m0) * (uint32_t)a.ld_x +
            copy_chunk16(lane) * 16u;
#pragma unroll
  for (int j = 0; j < WC; ++j)
    wo[j] = (uint32_t)min((j * WAVES + wave) * 8 + (lane >> 3), N - 1 - n0) * (uint32_t)K +
            copy_chunk16(lane) * 16u;
  const uint32_t lds = __builtin_amdgcn_readfirstlane(lds_address(smem) + wave * 1024);
  const int nkt = K / 128;
  auto issue = [&](int kt, int b) {
    const uint32_t base = lds + b * (SLOTS * 16);
#pragma unroll
    for (int j = 0; j < XC; ++j) copy_to_lds16_at(xs + kt * 128, xo[j], base + j * (WAVES * 1024));
#pragma unroll
    for (int j = 0; j < WC; ++j)
      copy_to_lds16_at(ws + kt * 128, wo[j], base + BM * 128 + j * (WAVES * 1024));
  };
  i32x4 acc[TI][TJ];
#pragma unroll
  for (int i = 0; i < TI; ++i)
#pragma unroll
    for (int j = 0; j < TJ; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
#pragma unroll
  for (int s = 0; s < STAGES - 1; ++s)
    if (s < nkt) issue(s, s);
  int b = 0;
  for (int kt = 0; kt < nkt; ++kt) {
    // This stage's copies are done; those of up to STAGES - 2 later ones may
    // not be.
    if (kt + STAGES - 2 < nkt)
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"((STAGES - 2) * (XC + WC)) : "memory");
    else
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();  // everyone's are, and the last stage is read out
    const u32x4* sx = smem + b * SLOTS;
    const u32x4* sw = sx + BM * 8;
    i32x4 fw[2][TI], fx[2][TJ];
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
#pragma unroll
      for (int i = 0; i < TI; ++i)
        fw[ks][i] = __builtin_bit_cast(i32x4, sw[swz16(wn0 + i * 16 + l16, ks * 4 + lq)]);
#pragma unroll
      for (int j = 0; j < TJ; ++j)
        fx[ks][j] = __builtin_bit_cast(i32x4, sx[swz16(wm0 + j * 16 + l16, ks * 4 + lq)]);
    }
    // The copies behind the reads, which would wait for their issue.
    const int free = b == 0 ? STAGES - 1 : b - 1;
    if (kt + STAGES - 1 < nkt) issue(kt + STAGES - 1, free);
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int i = 0; i < TI; ++i)
#pragma unroll
        for (int j = 0; j < TJ; ++j) acc[i][j] = mma(fw[ks][i], fx[ks][j], acc[i][j]);
    b = b == STAGES - 1 ? 0 : b + 1;
  }
  __syncthreads();  // the last stage is read out: the regions take its place
  u32x4* region = smem + wave * 256;
  auto slot16 = [&](int r, int c) { return region + r * 8 + c; };
  auto vec = [&](int v, int q) {
    const int n = min(n0 + wn0 + 4 * q, N - 4);
    return *reinterpret_cast<const float4*>((v ? a.bias : a.w_scale) + n);
  };
  auto scale = [&](int r) { return a.x_scale[min(m0 + wm0 + r, M - 1)]; };
  store_i8<TJ, TI, EPI>(acc, slot16, vec, scale, a, m0 + wm0, n0 + wn0, M, N, lane);
}

// A few tokens: the launch's time is a wave's chain and the stream of W.  16
// channels x 16 tokens a workgroup, whose eight waves take every eighth 128
// bytes of K straight from memory into registers, all loads of four turns in
// flight, and add up in LDS.
template <int EPI>
__global__ __launch_bounds__(512) void linear_i8_tokens_kernel(LinearI8 a, int M, int N, int K) {
  constexpr int WAVES = 8, BATCH = 4;
  __shared__ i32x4 part[WAVES][64];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l16 = lane & 15, lq = lane >> 4;
  const int n0 = blockIdx.x * 16, m0 = blockIdx.y * 16;
  const int8_t* wr = a.w + (int64_t)min(n0 + l16, N - 1) * K + lq * 16;
  const int8_t* xr = a.x + min(m0 + l16, M - 1) * a.ld_x + lq * 16;
  i32x4 acc = {0, 0, 0, 0};
  for (int k0 = wave * 128; k0 < K; k0 += BATCH * WAVES * 128) {
    i32x4 fw[BATCH][2], fx[BATCH][2];
#pragma unroll
    for (int q = 0; q < BATCH; ++q) {
      const int k = k0 + q * WAVES * 128;
      if (k >= K) break;
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        fw[q][s] = *reinterpret_cast<const i32x4*>(wr + k + s * 64);
        fx[q][s] = *reinterpret_cast<const i32x4*>(xr + k + s * 64);
      }
    }
#pragma unroll
    for (int q = 0; q < BATCH; ++q)
      if (k0 + q * WAVES * 128 < K) {
#pragma unroll
        for (int s = 0; s < 2; ++s) acc = mma(fw[q][s], fx[q][s], acc);
      }
  }
  part[wave][lane] = acc;
  __syncthreads();
  if (wave > 0) return;
  const int m = m0 + l16, n = n0 + 4 * lq;
  i32x4 v = part[0][lane];
#pragma unroll
  for (int w = 1; w < WAVES; ++w) v += part[w][lane];
  if (m >= M || n >= N) return;
  uint2 res = {0u, 0u};
  if constexpr (EPI == EPI_BIAS_RESIDUAL)
    res = *reinterpret_cast<const uint2*>(a.res + (int64_t)m * a.ld_res + n);
  *reinterpret_cast<uint2*>(a.y + (int64_t)m * a.ld_y + n) =
      finish_i8<EPI>(v, a.x_scale[m], *reinterpret_cast<const float4*>(a.w_scale + n),
                     *reinterpret_cast<const float4*>(a.bias + n), res);
}

// Few tiles and a long K: 64 tokens x 64 channels a workgroup, every fourth
// 128-byte stage of K in each of its four waves, which have two stages of LDS
// of their own and meet only to add up.
template <int EPI>
__global__ __launch_bounds__(256) void linear_i8_split_kernel(LinearI8 a, int M, int N, int K, int tiles_n,
                                                              int n_tiles) {
  constexpr int WAVES = 4, F = 4;   // fragments of 16 either way
  constexpr int SLOTS = 128 * 8;    // of a wave's stage
  __shared__ __attribute__((aligned(128))) u32x4 smem[WAVES * 2 * SLOTS];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l16 = lane & 15, lq = lane >> 4;
  int tm, tn;
  tile_coords<ORDER_ROW_GROUPS>(blockIdx.x, n_tiles, tiles_n, &tm, &tn);
  const int m0 = tm * 64, n0 = tn * 64;
  const int8_t* xs = a.x + (int64_t)m0 * a.ld_x;
  const int8_t* ws = a.w + (int64_t)n0 * K;
  // Copy j fills rows 8 j .. + 7 of either operand; rows past the matrix are
  // read clamped and never stored.
  uint32_t xo[8], wo[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int row = j * 8 + (lane >> 3);
    xo[j] = (uint32_t)min(row, M - 1 - m0) * (uint32_t)a.ld_x + copy_chunk16(lane) * 16u;
    wo[j] = (uint32_t)min(row, N - 1 - n0) * (uint32_t)K + copy_chunk16(lane) * 16u;
  }
  const uint32_t lds = __builtin_amdgcn_readfirstlane(lds_address(smem) + wave * (2 * SLOTS * 16));
  const int nkt = K / 128;
  auto issue = [&](int kt, int b) {
    const uint32_t base = lds + b * (SLOTS * 16);
#pragma unroll
    for (int j = 0; j < 8; ++j) copy_to_lds16_at(xs + kt * 128, xo[j], base + j * 1024);
#pragma unroll
    for (int j = 0; j < 8; ++j) copy_to_lds16_at(ws + kt * 128, wo[j], base + 8192 + j * 1024);
  };
  i32x4 acc[F][F];
#pragma unroll
  for (int i = 0; i < F; ++i)
#pragma unroll
    for (int j = 0; j < F; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
  int b = 0;
  if (wave < nkt) issue(wave, 0);
  for (int kt = wave; kt < nkt; kt += WAVES, b ^= 1) {
    if (kt + WAVES < nkt) {
      issue(kt + WAVES, b ^ 1);  // its last reads were waited for below
      asm volatile("s_waitcnt vmcnt(16)" ::: "memory");
    } else {
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    }
    const u32x4* sx = smem + (wave * 2 + b) * SLOTS;
    const u32x4* sw = sx + 64 * 8;
    i32x4 fw[2][F], fx[2][F];
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int i = 0; i < F; ++i) {
        fw[ks][i] = __builtin_bit_cast(i32x4, sw[swz16(i * 16 + l16, ks * 4 + lq)]);
        fx[ks][i] = __builtin_bit_cast(i32x4, sx[swz16(i * 16 + l16, ks * 4 + lq)]);
      }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int i = 0; i < F; ++i)
#pragma unroll
        for (int j = 0; j < F; ++j) acc[i][j] = mma(fw[ks][i], fx[ks][j], acc[i][j]);
  }
  __syncthreads();  // every wave has read its stages
#pragma unroll
  for (int i = 0; i < F; ++i)
#pragma unroll
    for (int j = 0; j < F; ++j)
      smem[((wave * F + j) * F + i) * 64 + lane] = __builtin_bit_cast(u32x4, acc[i][j]);
  __syncthreads();
  // Wave j finishes token fragment j.
  const int m = m0 + wave * 16 + l16;
  if (m >= M) return;
  const float sx = a.x_scale[m];
#pragma unroll
  for (int i = 0; i < F; ++i) {
    const int n = n0 + i * 16 + 4 * lq;
    if (n >= N) continue;
    i32x4 v = {0, 0, 0, 0};
#pragma unroll
    for (int w = 0; w < WAVES; ++w)
      v += __builtin_bit_cast(i32x4, smem[((w * F + wave) * F + i) * 64 + lane]);
    uint2 res = {0u, 0u};
    if constexpr (EPI == EPI_BIAS_RESIDUAL)
      res = *reinterpret_cast<const uint2*>(a.res + (int64_t)m * a.ld_res + n);
    *reinterpret_cast<uint2*>(a.y + (int64_t)m * a.ld_y + n) =
        finish_i8<EPI>(v, sx, *reinterpret_cast<const float4*>(a.w_scale + n),
                       *reinterpret_cast<const float4*>(a.bias + n), res);
  }
}

template <int WAVES_M, int WAVES_N, int TJ, int STAGES, int EPI>
void launch_ring(int64_t M, int N, int K, const LinearI8& a, hipStream_t stream) {
  constexpr int BM = WAVES_M * TJ * 16, BN = WAVES_N * 64;
  const int tiles_n = (N + BN - 1) / BN;
  const int n_tiles = (int)((M + BM - 1) / BM * tiles_n);
  hipLaunchKernelGGL((linear_i8_ring_kernel<WAVES_M, WAVES_N, TJ, STAGES, EPI>), dim3(n_tiles),
                     dim3(64 * WAVES_M * WAVES_N), 0, stream, a, (int)M, N, K, tiles_n, n_tiles);
}

template <int WAVES_M, int WAVES_N, int TI, int J0, int EPI>
void launch_wide(int64_t M, int N, int K, const LinearI8& a, int n_cus, hipStream_t stream) {
  constexpr int BM = WAVES_M * 16 * (J0 + 2);
  const int tiles_n = N / 256;
  const int n_tiles = (int)((M + BM - 1) / BM * tiles_n);
  hipLaunchKernelGGL((linear_i8_wide_kernel<WAVES_M, WAVES_N, TI, J0, 2, EPI>),
                     dim3(std::min(n_tiles, n_cus)), dim3(512), 0, stream, a, (int)M, K, tiles_n, n_tiles);
}

// Which kernel: the one of the least time by a model of its rounds.  A launch
// of `tiles` on n_cus CUs that hold `per_cu` of them at a time has c = tiles
// per CU and r = c / per_cu rounds (each rounded up) and takes, with s = K /
// 128 stages,
//   base + r (round + round_s s) + c (tile + tile_s s) us:
// what a round's latencies cost, and what tiles that share a CU cost each
// other.  Fitted to 1,275 launches of 250 shapes (M = 1 .. 60,000, N = 128 ..
// 4096, K = 128 .. 4096, each under every kernel but the split one): 5 to 9 %
// of the time in the mean square, and the kernel taken is 0.9 % slower than
// the shape's best in the mean, 25 % at worst.  Measured (us, tokens / 64 x 64 / 64 x 128 / 128 x
// 128 / 192 x 256 / 256 x 256):
//   N = 768, K = 768    M = 1 2.7 / 4.2 / 4.6 / 6.3 / 10.4 / 12.5
//                       1024 11.1 / 4.7 / 5.1 / 6.8 / 11.1 / 13.2
//                       13,579 110 / 18.7 / 16.4 / 16.6 / 13.2 / 14.7
//   N = 2304, K = 768   M = 1500 39.4 / 8.8 / 7.0 / 8.0 / 11.7 / 14.0
//                       6000 145 / 23.7 / 21.9 / 18.2 / 22.0 / 16.2
//   N = 1024, K = 4096  M = 1 4.2 / 11.2 / 13.1 / 18.9 / 32.6 / 40.2
//                       20,000 1,091 / 119 / 101 / 88.1 / 78.5 / 90.0,
// and with K split over a tile's waves against the 64 x 64 ring: N = 1024, K =
// 4096 M = 200 8.6 / 11.5, 1024 10.1 / 12.4, 1500 (two tiles on a CU) 17.3 /
// 14.7; K = 768 M = 777 5.1 / 4.6.
enum Kernel { TOKENS, SPLIT_64x64, RING_64x64, RING_64x128, RING_128x128, WIDE_192, WIDE_256, KERNELS };
struct Cost {
  int rows, cols, per_cu;
  double base, round, round_s, tile, tile_s;
};
constexpr Cost COSTS[KERNELS] = {
    {16, 16, 3, 2.1, 0.09, 0.0, 0.08, 0.10},   {64, 64, 1, 0.4, 0.0, 0.0, 3.60, 0.18},
    {64, 64, 3, 2.1, 0.62, 0.14, 0.35, 0.12},  {64, 128, 2, 1.6, 1.02, 0.08, 0.48, 0.25},
    {128, 128, 2, 0.6, 2.39, 0.17, 0.83, 0.36}, {192, 256, 1, 0.2, 0.0, 0.0, 5.50, 0.91},
    {256, 256, 1, 0.0, 0.0, 0.0, 6.70, 1.13},
};

double kernel_us(Kernel k, int64_t M, int N, int K, int n_cus) {
  const Cost& q = COSTS[k];
  auto up = [](int64_t a, int64_t b) { return (a + b - 1) / b; };
  const int64_t c = up(up(M, q.rows) * up(N, q.cols), n_cus), r = up(c, q.per_cu);
  const double s = K / 128;
  return q.base + (double)r * (q.round + q.round_s * s) + (double)c * (q.tile + q.tile_s * s);
}

// The best of kernels 0 .. n - 1.
Kernel best_kernel(int n, int64_t M, int N, int K, int n_cus, double* us) {
  Kernel best = RING_64x64;
  *us = kernel_us(best, M, N, K, n_cus);
  for (int i = 0; i < n; ++i) {
    if (i == TOKENS && M > 16 * 65535) continue;  // its grid's second dimension
    const double t = kernel_us((Kernel)i, M, N, K, n_cus);
    if (t < *us) {
      *us = t;
      best = (Kernel)i;
    }
  }
  return best;
}

// The wide tiles take whole 256 channels; what is left of N goes to the best
// of the others in a launch of its own.
Kernel choose(int64_t M, int N, int K, int n_cus) {
  double us;
  const Kernel k = best_kernel(WIDE_192, M, N, K, n_cus, &us);
  if (N < 256) return k;
  double rest = 0;
  if (N % 256) best_kernel(WIDE_192, M, N % 256, K, n_cus, &rest);
  const double w192 = kernel_us(WIDE_192, M, N & ~255, K, n_cus) + rest;
  const double w256 = kernel_us(WIDE_256, M, N & ~255, K, n_cus) + rest;
  if (std::min(w192, w256) >= us) return k;
  return w192 < w256 ? WIDE_192 : WIDE_256;
}

template <int EPI>
hipError_t launch(int64_t M, int N, int K, const LinearI8& a, int n_cus, hipStream_t stream) {
  switch (choose(M, N, K, n_cus)) {
    case TOKENS:
      hipLaunchKernelGGL((linear_i8_tokens_kernel<EPI>), dim3((N + 15) / 16, (unsigned)((M + 15) / 16)),
                         dim3(512), 0, stream, a, (int)M, N, K);
      return hipGetLastError();
    case SPLIT_64x64: {
      const int tiles_n = (N + 63) / 64, n_tiles = (int)((M + 63) / 64 * tiles_n);
      hipLaunchKernelGGL((linear_i8_split_kernel<EPI>), dim3(n_tiles), dim3(256), 0, stream, a, (int)M, N, K,
                         tiles_n, n_tiles);
      return hipGetLastError();
    }
    case RING_64x64: launch_ring<2, 1, 2, 3, EPI>(M, N, K, a, stream); return hipGetLastError();
    case RING_64x128: launch_ring<2, 2, 2, 3, EPI>(M, N, K, a, stream); return hipGetLastError();
    case RING_128x128: launch_ring<2, 2, 4, 2, EPI>(M, N, K, a, stream); return hipGetLastError();
    case WIDE_192: launch_wide<2, 4, 4, 4, EPI>(M, N, K, a, n_cus, stream); break;
    default: launch_wide<4, 2, 8, 2, EPI>(M, N, K, a, n_cus, stream); break;
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || N % 256 == 0) return e;
  const int cols = N & ~255;
  LinearI8 rest = a;
  rest.w += (int64_t)cols * K;
  rest.w_scale += cols;
  rest.bias += cols;
  if (rest.res) rest.res += cols;
  rest.y += cols;
  return launch<EPI>(M, N - cols, K, rest, n_cus, stream);
}

}  // namespace

int linear_i8_tile(int64_t M, int N, int K, int n_cus) {
  const Cost& q = COSTS[choose(std::min<int64_t>(M, 1 << 24), N, K, n_cus)];
  return q.rows << 16 | q.cols;
}

// Rows in launches of at most 2^24, so that row numbers and grids stay well
// inside 32 bits.
hipError_t launch_linear_i8(int64_t M, int N, int K, int epi, const LinearI8& a, int n_cus,
                            hipStream_t stream) {
  constexpr int64_t MOST = 1 << 24;
  for (int64_t m = 0; m < M; m += MOST) {
    const int64_t rows = std::min(MOST, M - m);
    LinearI8 part = a;
    part.x += m * a.ld_x;
    part.x_scale += m;
    if (part.res) part.res += m * a.ld_res;
    part.y += m * a.ld_y;
    const hipError_t e = epi == EPI_BIAS        ? launch<EPI_BIAS>(rows, N, K, part, n_cus, stream)
                         : epi == EPI_BIAS_GELU ? launch<EPI_BIAS_GELU>(rows, N, K, part, n_cus, stream)
                                                : launch<EPI_BIAS_RESIDUAL>(rows, N, K, part, n_cus, stream);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace surge
