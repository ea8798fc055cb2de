// Row kernels of a reader's block (gfx950): quantizing rows to int8 with a
// scale per token, and the norms after a block and before the next one fused
// with the gate, the residual scale and the quantizer.
//
// A row is held in registers by LANES lanes (a part of a wave, a wave, or the
// four waves of a workgroup), CH chunks of 8 features a lane, chunk c = j
// LANES + lane: every load and store of a row is contiguous.  So each input
// is read once, the mean and the variance are two passes over registers (no
// E[v^2] - mean^2 cancellation), and all sums are fp32.
#include <math.h>

#include <algorithm>

#include "device_common.h"
#include "reader.h"

namespace surge {
namespace {

constexpr int BLOCK = 256;

enum Reduce { SUM, MAX };

// Sum or maximum over the LANES lanes of a row.  LANES = 256: the workgroup,
// through `lds` (4 floats, one use per call between two barriers).
template <int LANES, Reduce OP>
__device__ __forceinline__ float row_reduce(float v, float* lds) {
#pragma unroll
  for (int o = (LANES < 64 ? LANES : 64) / 2; o >= 1; o >>= 1) {
    const float w = __shfl_xor(v, o, 64);
    v = OP == SUM ? v + w : fmaxf(v, w);
  }
  if constexpr (LANES == 256) {
    __syncthreads();  // the previous use has been read
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = OP == SUM ? (lds[0] + lds[1]) + (lds[2] + lds[3])
                  : fmaxf(fmaxf(lds[0], lds[1]), fmaxf(lds[2], lds[3]));
  }
  return v;
}

// A row's scale and the factor that its values are multiplied by before
// rounding.  The largest magnitude is clamped to 2^-100, so that neither
// overflows nor loses bits as a subnormal; a row of zeros gets the scale of
// the clamp.
struct RowScale {
  float inv, scale;
};
__device__ __forceinline__ RowScale row_scale(float amax) {
  const float a = fmaxf(amax, 0x1p-100f);
  return {127.0f / a, a / 127.0f};
}

// The largest magnitude of 8 values, infinity where one is not finite (fmaxf
// would drop a NaN).
__device__ __forceinline__ float amax8(const float* f, float m) {
#pragma unroll
  for (int i = 0; i < 8; ++i) m = fabsf(f[i]) <= 3.4028234e38f ? fmaxf(m, fabsf(f[i])) : INFINITY;
  return m;
}

__device__ __forceinline__ uint2 quantize8(const float* f, float inv) {
  uint32_t w[2] = {0u, 0u};
#pragma unroll
  for (int i = 0; i < 8; ++i)
    w[i >> 2] |= (uint32_t)((int)rintf(f[i] * inv) & 0xff) << (8 * (i & 3));
  return {w[0], w[1]};
}

// What surge.h calls a row that cannot be quantized: zeros under a NaN scale.
__device__ __forceinline__ RowScale poisoned() { return {0.0f, NAN}; }

template <int LANES, int CH>
__global__ __launch_bounds__(BLOCK) void quantize_rows_kernel(int64_t M, int K,
                                                              const uint16_t* x, int64_t ld_x,
                                                              int8_t* q, int64_t ld_q,
                                                              float* scale) {
  constexpr int ROWS = BLOCK / LANES;
  __shared__ float lds[4];
  const int lane = threadIdx.x % LANES;
  const int64_t m = (int64_t)blockIdx.x * ROWS + threadIdx.x / LANES;
  if (m >= M) return;  // LANES = 256: the whole workgroup
  const int chunks = K / 8, padded = (K + 127) / 128 * 16;
  const uint16_t* xr = x + m * ld_x;
  uint4 raw[CH];
#pragma unroll
  for (int j = 0; j < CH; ++j) {
    const int c = j * LANES + lane;
    raw[j] = c < chunks ? *reinterpret_cast<const uint4*>(xr + 8 * c) : uint4{0u, 0u, 0u, 0u};
  }
  float amax = 0.0f, f[8];
#pragma unroll
  for (int j = 0; j < CH; ++j) {
    unpack8(raw[j], f);
    amax = amax8(f, amax);
  }
  amax = row_reduce<LANES, MAX>(amax, lds);
  const bool bad = amax == INFINITY;
  const RowScale s = bad ? poisoned() : row_scale(amax);
#pragma unroll
  for (int j = 0; j < CH; ++j) {
    const int c = j * LANES + lane;
    unpack8(raw[j], f);
    if (c < padded)
      *reinterpret_cast<uint2*>(q + m * ld_q + 8 * c) = bad ? uint2{0u, 0u} : quantize8(f, s.inv);
  }
  if (lane == 0) scale[m] = s.scale;
}

// v <- the row's norm of v.  Chunks past the row hold 0 and stay out of the
// variance.
template <int LANES, int CH, bool RMS>
__device__ __forceinline__ void row_norm(float (&v)[CH][8], int lane, int chunks, int d, float eps,
                                         const float* gamma, const float* beta, float* lds) {
  const float inv_d = 1.0f / (float)d;
  float mean = 0.0f, sq = 0.0f;
  if constexpr (!RMS) {
    float s = 0.0f;
#pragma unroll
    for (int j = 0; j < CH; ++j)
#pragma unroll
      for (int i = 0; i < 8; ++i) s += v[j][i];
    mean = row_reduce<LANES, SUM>(s, lds) * inv_d;
  }
#pragma unroll
  for (int j = 0; j < CH; ++j)
    if (j * LANES + lane < chunks) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        v[j][i] -= mean;
        sq = fmaf(v[j][i], v[j][i], sq);
      }
    }
  const float rstd = 1.0f / sqrtf(fmaf(row_reduce<LANES, SUM>(sq, lds), inv_d, eps));
#pragma unroll
  for (int j = 0; j < CH; ++j) {
    const int c = j * LANES + lane;
    if (c < chunks) {
      const float4* g = reinterpret_cast<const float4*>(gamma + 8 * c);
      const float4 g0 = g[0], g1 = g[1];
      const float gg[8] = {g0.x, g0.y, g0.z, g0.w, g1.x, g1.y, g1.z, g1.w};
#pragma unroll
      for (int i = 0; i < 8; ++i) v[j][i] *= rstd * gg[i];
      if (beta) {
        const float4* b = reinterpret_cast<const float4*>(beta + 8 * c);
        const float4 b0 = b[0], b1 = b[1];
        const float bb[8] = {b0.x, b0.y, b0.z, b0.w, b1.x, b1.y, b1.z, b1.w};
#pragma unroll
        for (int i = 0; i < 8; ++i) v[j][i] += bb[i];
      }
    }
  }
}

template <int LANES, int CH, bool RMS>
__global__ __launch_bounds__(BLOCK) void block_norm_kernel(int64_t M, int d, BlockNorm a) {
  constexpr int ROWS = BLOCK / LANES;
  __shared__ float lds[4];
  const int lane = threadIdx.x % LANES;
  const int64_t m = (int64_t)blockIdx.x * ROWS + threadIdx.x / LANES;
  if (m >= M) return;  // LANES = 256: the whole workgroup
  const int chunks = d / 8;
  const uint4 zero = {0u, 0u, 0u, 0u};
  uint4 xr[CH], br[CH], gr[CH];
#pragma unroll
  for (int j = 0; j < CH; ++j) {
    const int c = j * LANES + lane;
    const bool in = c < chunks;
    xr[j] = in ? *reinterpret_cast<const uint4*>(a.x + m * a.ld_x + 8 * c) : zero;
    br[j] = in && a.block ? *reinterpret_cast<const uint4*>(a.block + m * a.ld_block + 8 * c) : zero;
    gr[j] = in && a.gate_rows ? *reinterpret_cast<const uint4*>(a.gate_rows + m * a.ld_gate + 8 * c)
                              : zero;
  }
  float v[CH][8];
#pragma unroll
  for (int j = 0; j < CH; ++j) unpack8(br[j], v[j]);
  if (a.post_gamma)
    row_norm<LANES, CH, RMS>(v, lane, chunks, d, a.eps, a.post_gamma, a.post_beta, lds);
#pragma unroll
  for (int j = 0; j < CH; ++j) {
    const int c = j * LANES + lane;
    float f[8];
    if (a.gate_rows) {
      unpack8(gr[j], f);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[j][i] *= f[i];
    }
    if (a.gate && c < chunks) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[j][i] *= a.gate[8 * c + i];
    }
    unpack8(xr[j], f);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[j][i] = fmaf(a.res_scale, f[i], v[j][i]);
    if (a.y && c < chunks) *reinterpret_cast<uint4*>(a.y + m * a.ld_y + 8 * c) = pack8(v[j]);
  }
  if (!a.z && !a.zq) return;
  // The next block's norm reads the stream before its rounding to bf16.
  row_norm<LANES, CH, RMS>(v, lane, chunks, d, a.eps, a.pre_gamma, a.pre_beta, lds);
  if (a.z) {
#pragma unroll
    for (int j = 0; j < CH; ++j) {
      const int c = j * LANES + lane;
      if (c < chunks) *reinterpret_cast<uint4*>(a.z + m * a.ld_z + 8 * c) = pack8(v[j]);
    }
  }
  if (a.zq) {
    float amax = 0.0f;
#pragma unroll
    for (int j = 0; j < CH; ++j) amax = amax8(v[j], amax);
    amax = row_reduce<LANES, MAX>(amax, lds);
    const bool bad = amax == INFINITY;
    const RowScale s = bad ? poisoned() : row_scale(amax);
    const int padded = (d + 127) / 128 * 16;
#pragma unroll
    for (int j = 0; j < CH; ++j) {
      const int c = j * LANES + lane;
      if (c < padded)
        *reinterpret_cast<uint2*>(a.zq + m * a.ld_zq + 8 * c) =
            bad ? uint2{0u, 0u} : quantize8(v[j], s.inv);
    }
    if (lane == 0) a.zq_scale[m] = s.scale;
  }
}

}  // namespace

// The fewest lanes whose 4 chunks (8 beyond 8192 features) hold a padded row:
// short rows share a wave, rows beyond 2048 features take a workgroup.
hipError_t launch_quantize_rows(int64_t M, int K, const uint16_t* x, int64_t ld_x, int8_t* q,
                                int64_t ld_q, float* scale, hipStream_t stream) {
  if (M <= 0) return hipSuccess;
  const int n = (int)i8_columns(K) / 8;
#define SURGE_LAUNCH(LANES, CH)                                                               \
  hipLaunchKernelGGL((quantize_rows_kernel<LANES, CH>),                                       \
                     dim3((unsigned)((M + BLOCK / LANES - 1) / (BLOCK / LANES))), dim3(BLOCK), \
                     0, stream, M, K, x, ld_x, q, ld_q, scale)
  if (n <= 64)
    SURGE_LAUNCH(16, 4);
  else if (n <= 128)
    SURGE_LAUNCH(32, 4);
  else if (n <= 256)
    SURGE_LAUNCH(64, 4);
  else if (n <= 1024)
    SURGE_LAUNCH(256, 4);
  else
    SURGE_LAUNCH(256, 8);
#undef SURGE_LAUNCH
  return hipGetLastError();
}

hipError_t launch_block_norm(int64_t M, int d, bool rms, const BlockNorm& a, hipStream_t stream) {
  if (M <= 0) return hipSuccess;
  const int n = (int)i8_columns(d) / 8;
#define SURGE_LAUNCH_KIND(LANES, CH, RMS)                                                     \
  hipLaunchKernelGGL((block_norm_kernel<LANES, CH, RMS>),                                     \
                     dim3((unsigned)((M + BLOCK / LANES - 1) / (BLOCK / LANES))), dim3(BLOCK), \
                     0, stream, M, d, a)
#define SURGE_LAUNCH(LANES, CH)       \
  if (rms)                            \
    SURGE_LAUNCH_KIND(LANES, CH, true); \
  else                                \
    SURGE_LAUNCH_KIND(LANES, CH, false)
  if (n <= 64) {
    SURGE_LAUNCH(16, 4);
  } else if (n <= 128) {
    SURGE_LAUNCH(32, 4);
  } else if (n <= 256) {
    SURGE_LAUNCH(64, 4);
  } else {
    SURGE_LAUNCH(256, 4);
  }
#undef SURGE_LAUNCH
#undef SURGE_LAUNCH_KIND
  return hipGetLastError();
}

}  // namespace surge
