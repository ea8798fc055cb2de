// Linear layers in 8-bit integers (gfx950): y = epi(sx[m] sw[n] (X W^T)[m][n]
// + b[n]), X [M, K] int8 with a scale per token, W [N, K] int8 with a scale
// per output channel.  The products are summed exactly in 32-bit integers
// (K <= 65,536 of at most 2^14 each), so only the finish rounds: one
// conversion to fp32, two products, the bias, GELU or residual, and bf16.
//
// A row's 128 bytes of a K stage are laid out as the bf16 layers lay out
// their 64 values: a fragment of a 16x16x64 MFMA is 16 rows x four 16-byte
// chunks, read from LDS rows whose chunk c of row r sits at c ^ (r & 7).
#include <algorithm>

#include "linear_common.h"
#include "reader.h"

namespace surge {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));

// Four waves of 64 x 64; two stages of (128 + 128) rows x 128 bytes.
template <int EPI>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2))) void linear_i8_kernel(
    LinearI8 a, int M, int N, int K, int tiles_n, int n_tiles) {
  constexpr int BM = 128, BN = 128;
  constexpr int SLOTS = (BM + BN) * 8;
  __shared__ u32x4 smem[2][SLOTS];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l16 = lane & 15, lq = lane >> 4;
  const int wn0 = (wave & 1) * 64, wm0 = (wave >> 1) * 64;
  int tm, tn;
  tile_coords<ORDER_ROW_GROUPS>(blockIdx.x, n_tiles, tiles_n, &tm, &tn);
  const int m0 = tm * BM, n0 = tn * BN;
  const int8_t* xs = a.x + (int64_t)m0 * a.ld_x;
  const int8_t* ws = a.w + (int64_t)n0 * K;
  // Copy j of wave w fills rows (4 j + w) 8 .. + 7 of either operand; rows
  // past the matrix are read clamped and never stored.
  uint32_t xo[4], wo[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int row = (j * 4 + wave) * 8 + (lane >> 3);
    xo[j] = (uint32_t)min(row, M - 1 - m0) * (uint32_t)a.ld_x + copy_chunk16(lane) * 16u;
    wo[j] = (uint32_t)min(row, N - 1 - n0) * (uint32_t)K + copy_chunk16(lane) * 16u;
  }
  const uint32_t lds = __builtin_amdgcn_readfirstlane(lds_address(smem) + wave * 1024);
  auto issue = [&](int kt, int b) {
    const uint32_t base = lds + b * SLOTS * 16;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      copy_to_lds16_at(xs + kt * 128, xo[j], base + j * 4096);
      copy_to_lds16_at(ws + kt * 128, wo[j], base + BM * 128 + j * 4096);
    }
  };
  i32x4 acc[4][4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
  const int nkt = K / 128;
  issue(0, 0);
  for (int kt = 0; kt < nkt; ++kt) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (kt + 1 < nkt) issue(kt + 1, (kt + 1) & 1);
    const u32x4* sx = smem[kt & 1];
    const u32x4* sw = sx + BM * 8;
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      i32x4 fw[4], fx[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        fw[i] = __builtin_bit_cast(i32x4, sw[swz16(wn0 + i * 16 + l16, ks * 4 + lq)]);
        fx[i] = __builtin_bit_cast(i32x4, sx[swz16(wm0 + i * 16 + l16, ks * 4 + lq)]);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fw[i], fx[j], acc[i][j], 0, 0, 0);
    }
    // This stage's reads are done before the next but one is copied over it.
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __syncthreads();
  }
  // Lane: features n .. n + 3 of token m; N is a multiple of 8.
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int m = m0 + wm0 + j * 16 + l16;
    if (m >= M) continue;
    const float sx = a.x_scale[m];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int n = n0 + wn0 + i * 16 + 4 * lq;
      if (n >= N) continue;
      const float4 sw = *reinterpret_cast<const float4*>(a.w_scale + n);
      const float4 bb = *reinterpret_cast<const float4*>(a.bias + n);
      const i32x4 v = acc[i][j];
      const float s[4] = {(float)v[0] * sx * sw.x, (float)v[1] * sx * sw.y, (float)v[2] * sx * sw.z,
                          (float)v[3] * sx * sw.w};
      uint2 res = {0u, 0u};
      if constexpr (EPI == EPI_BIAS_RESIDUAL)
        res = *reinterpret_cast<const uint2*>(a.res + (int64_t)m * a.ld_res + n);
      *reinterpret_cast<uint2*>(a.y + (int64_t)m * a.ld_y + n) =
          finish4<EPI>(s, bb, bb, bb, bb, 0.0f, 0.0f, res);
    }
  }
}

}  // namespace

hipError_t launch_linear_i8(int64_t M, int N, int K, int epi, const LinearI8& a, int n_cus,
                            hipStream_t stream) {
  if (M <= 0) return hipSuccess;
  const int tiles_n = (N + 127) / 128;
  const int64_t n_tiles = (M + 127) / 128 * tiles_n;
  if (n_tiles > INT32_MAX) return hipErrorInvalidValue;
  const dim3 grid((unsigned)n_tiles), block(256);
#define SURGE_LAUNCH(E) \
  hipLaunchKernelGGL((linear_i8_kernel<E>), grid, block, 0, stream, a, (int)M, N, K, tiles_n, (int)n_tiles)
  switch (epi) {
    case EPI_BIAS: SURGE_LAUNCH(EPI_BIAS); break;
    case EPI_BIAS_GELU: SURGE_LAUNCH(EPI_BIAS_GELU); break;
    default: SURGE_LAUNCH(EPI_BIAS_RESIDUAL); break;
  }
#undef SURGE_LAUNCH
  return hipGetLastError();
}

}  // namespace surge
