// Row kernels of a reader's block (gfx950): quantizing rows to int8 with a
// scale per token, and the norms after a block and before the next one fused
// with the gate, the residual scale and the quantizer.
//
// A row is held in registers by LANES lanes (16 or 32 of a wave, a wave, or
// the four or eight waves of a workgroup), CH chunks of 8 features a lane,
// chunk c = j LANES + lane: every load and store of a row is contiguous.  So
// each input is read once, the mean and the variance are two passes over registers (no
// E[v^2] - mean^2 cancellation), and all sums are fp32.
//
// What bounds them, measured: memory.  200,003 rows of 1024 with gate rows take
// 340 to 350 us (5.8 to 6.0 TB/s for 2.05 GB), quantizing 200,003 rows of 4096
// 366 to 400 us (6.1 to 6.7 TB/s), where a large copy reaches 4.8.  Rows of a few
// thousand: 13,579 of 768 to int8 21 to 22 us (3.4 TB/s), a wave's five rows one
// after the other at three waves per SIMD (148 registers).  Small calls: 64 rows
// of 1024 4 us, the chain of a row's loads and its four reductions.
#include <float.h>
#include <math.h>

#include <algorithm>

#include "device_common.h"
#include "reader.h"

namespace surge {
namespace {

// Threads of a workgroup: of several rows, or the lanes of one.
constexpr int block_of(int lanes) { return lanes > 256 ? lanes : 256; }

enum Reduce { SUM, MAX };

template <Reduce OP>
__device__ __forceinline__ float combine(float a, float b) {
  return OP == SUM ? a + b : fmaxf(a, b);
}

// v combined with its value in another lane of the same 16 (a DPP control).
template <Reduce OP, int CTRL>
__device__ __forceinline__ float with_lane(float v) {
  return combine<OP>(v, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), CTRL, 0xf, 0xf, true)));
}

// Sum or maximum over the LANES lanes of a row, all lanes of the wave active.
// Exchanges in registers: a reduction over a wave is six of them, where one
// through LDS is six LDS latencies.  LANES > 64: the workgroup, through one
// of two LDS slots by turns, so that one barrier a call is enough.
template <int LANES, Reduce OP>
__device__ __forceinline__ float row_reduce(float v, float (&lds)[2][16], int& turn) {
  v = with_lane<OP, 0xB1>(v);   // lane ^ 1
  v = with_lane<OP, 0x4E>(v);   // lane ^ 2
  v = with_lane<OP, 0x141>(v);  // 7 - lane of 8
  v = with_lane<OP, 0x140>(v);  // 15 - lane of 16
  if constexpr (LANES >= 32) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = combine<OP>(__uint_as_float(r[0]), __uint_as_float(r[1]));
  }
  if constexpr (LANES >= 64) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = combine<OP>(__uint_as_float(r[0]), __uint_as_float(r[1]));
  }
  if constexpr (LANES > 64) {
    if ((threadIdx.x & 63) == 0) lds[turn][threadIdx.x >> 6] = v;
    __syncthreads();
    v = lds[turn][0];
#pragma unroll
    for (int w = 1; w < LANES / 64; ++w) v = combine<OP>(v, lds[turn][w]);
    turn ^= 1;
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

// Rows are touched once: loads and stores that leave the caches to others (an
// L2 that keeps the outputs writes them back beside the next reads: 200,003
// rows of 1024 with gate rows 428 -> 340 us, of 768 418 -> 302).
__device__ __forceinline__ uint4 load16(const uint16_t* p) {
  return __builtin_bit_cast(uint4, __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p)));
}
__device__ __forceinline__ void store16(uint16_t* p, uint4 v) {
  __builtin_nontemporal_store(__builtin_bit_cast(u32x4, v), reinterpret_cast<u32x4*>(p));
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

// A row that cannot be quantized: zeros under a NaN scale.
__device__ __forceinline__ RowScale poisoned() { return {0.0f, NAN}; }

// Quantizes a row of fp32 values, chunk(j, f) giving its chunks.
template <int LANES, int CH, class Chunk>
__device__ __forceinline__ void store_quantized(Chunk chunk, int lane, int padded, bool store, int8_t* q,
                                                float* scale, float (&lds)[2][16], int& turn) {
  float amax = 0.0f, f[8];
#pragma unroll
  for (int j = 0; j < CH; ++j) {
    chunk(j, f);
    amax = amax8(f, amax);
  }
  amax = row_reduce<LANES, MAX>(amax, lds, turn);
  const bool bad = amax == INFINITY;
  const RowScale s = bad ? poisoned() : row_scale(amax);
#pragma unroll
  for (int j = 0; j < CH; ++j) {
    const int c = j * LANES + lane;
    chunk(j, f);
    if (store && c < padded)
      *reinterpret_cast<uint2*>(q + 8 * c) = bad ? uint2{0u, 0u} : quantize8(f, s.inv);
  }
  if (store && lane == 0) *scale = s.scale;
}

template <int LANES, int CH>
__global__ __launch_bounds__(block_of(LANES)) void quantize_rows_kernel(int64_t M, int K,
                                                              const uint16_t* x, int64_t ld_x,
                                                              int8_t* q, int64_t ld_q,
                                                              float* scale) {
  constexpr int ROWS = block_of(LANES) / LANES;
  __shared__ float lds[2][16];
  int turn = 0;
  const int lane = threadIdx.x % LANES;
  const int chunks = K / 8;
  for (int64_t m0 = (int64_t)blockIdx.x * ROWS; m0 < M; m0 += (int64_t)gridDim.x * ROWS) {
    const int64_t m = m0 + threadIdx.x / LANES;
    const uint16_t* xr = x + min(m, M - 1) * ld_x;
    uint4 raw[CH];
#pragma unroll
    for (int j = 0; j < CH; ++j) {
      const int c = j * LANES + lane;
      raw[j] = c < chunks ? load16(xr + 8 * c) : uint4{0u, 0u, 0u, 0u};
    }
    store_quantized<LANES, CH>([&](int j, float* f) { unpack8(raw[j], f); }, lane, (K + 127) / 128 * 16,
                               m < M, q + m * ld_q, scale + m, lds, turn);
  }
}

// 8 consecutive features of an fp32 vector, or `none` where there is none.
__device__ __forceinline__ void load8(const float* v, int c, bool in, float none, float (&f)[8]) {
  float4 a = {none, none, none, none}, b = a;
  if (v && in) {
    a = reinterpret_cast<const float4*>(v + 8 * c)[0];
    b = reinterpret_cast<const float4*>(v + 8 * c)[1];
  }
  const float t[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = t[i];
}

// The factor and the summand of a lane's features: gamma and beta of a norm,
// for the norm after the block times the gate.
template <int LANES, int CH>
struct Affine {
  float g[CH][8], b[CH][8];
  __device__ __forceinline__ void load(const float* gamma, const float* beta, const float* gate, int lane,
                                       int chunks) {
#pragma unroll
    for (int j = 0; j < CH; ++j) {
      const int c = j * LANES + lane;
      load8(gamma, c, c < chunks, 1.0f, g[j]);
      load8(beta, c, c < chunks, 0.0f, b[j]);
      if (gate) {
        float f[8];
        load8(gate, c, c < chunks, 0.0f, f);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          g[j][i] *= f[i];
          // A beta of 0, or none, stays 0 under an infinite gate.
          b[j][i] = b[j][i] == 0.0f ? 0.0f : b[j][i] * f[i];
        }
      }
    }
  }
};

// v <- (v - mean) / sqrt(var + eps) over the row, or v / sqrt(mean v^2 + eps).
// Chunks past the row hold 0 and stay out of the variance.
template <int LANES, int CH, bool RMS>
__device__ __forceinline__ void normalise(float (&v)[CH][8], int lane, int chunks, float inv_d, float eps,
                                          float (&lds)[2][16], int& turn) {
  float mean = 0.0f, sq = 0.0f;
  if constexpr (!RMS) {
    float s = 0.0f;
#pragma unroll
    for (int j = 0; j < CH; ++j)
#pragma unroll
      for (int i = 0; i < 8; ++i) s += v[j][i];
    mean = row_reduce<LANES, SUM>(s, lds, turn) * inv_d;
  }
#pragma unroll
  for (int j = 0; j < CH; ++j)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if constexpr (!RMS) v[j][i] = j * LANES + lane < chunks ? v[j][i] - mean : 0.0f;
      sq = fmaf(v[j][i], v[j][i], sq);
    }
  float ms = fmaf(row_reduce<LANES, SUM>(sq, lds, turn), inv_d, eps);
  // Squares above the largest float, or near the least where eps is too: once more
  // with the row times a power of 2, which leaves v / sqrt(ms) what it is.  (The
  // lanes of a row agree, and a wave or a workgroup takes the branch as one.)
  if (__any(!(ms >= 0x1p-100f && ms <= FLT_MAX))) {
    const float by = ms > FLT_MAX ? 0x1p-80f : ms < 0x1p-100f ? 0x1p80f : 1.0f;
    sq = 0.0f;
#pragma unroll
    for (int j = 0; j < CH; ++j)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        v[j][i] *= by;
        sq = fmaf(v[j][i], v[j][i], sq);
      }
    ms = fmaf(row_reduce<LANES, SUM>(sq, lds, turn), inv_d, eps * by * by);
  }
  const float rstd = 1.0f / sqrtf(ms);
#pragma unroll
  for (int j = 0; j < CH; ++j)
#pragma unroll
    for (int i = 0; i < 8; ++i) v[j][i] *= rstd;
}

// A lane group works through `turns` rows with the vectors in registers and
// reads the next row while it works on one; the rows of a workgroup are
// consecutive (a grid's stride between them: 341 -> 383 us for 200,003 rows of
// 1024 with gate rows).
template <int LANES, int CH, bool RMS>
__global__ __launch_bounds__(block_of(LANES)) void block_norm_kernel(int64_t M, int d, int turns, BlockNorm a) {
  constexpr int ROWS = block_of(LANES) / LANES;               // rows of a workgroup at a time
  constexpr int PER = LANES < 64 ? 64 / LANES : 1;  // and of a wave
  __shared__ float lds[2][16];
  int turn = 0;
  const int lane = threadIdx.x % LANES;
  const int sub = threadIdx.x / LANES;
  const int chunks = d / 8;
  const float inv_d = 1.0f / (float)d;
  const bool norm = a.z || a.zq;
  struct Row {
    uint4 x[CH], b[CH], g[CH];
  };
  auto read = [&](int64_t m, Row& r) {
    const uint4 zero = {0u, 0u, 0u, 0u};
    m = min(m, M - 1);
#pragma unroll
    for (int j = 0; j < CH; ++j) {
      const int c = j * LANES + lane;
      const bool in = c < chunks;
      r.x[j] = in ? load16(a.x + m * a.ld_x + 8 * c) : zero;
      r.b[j] = in && a.block ? load16(a.block + m * a.ld_block + 8 * c) : zero;
      r.g[j] = in && a.gate_rows ? load16(a.gate_rows + m * a.ld_gate + 8 * c)
                                 : zero;
    }
  };
  // The rows of this wave (of the workgroup) at each turn start at m0.
  const int64_t first = (int64_t)blockIdx.x * (ROWS * turns) + sub / PER * PER;
  const int64_t step = ROWS, end = min(M, ((int64_t)blockIdx.x + 1) * (ROWS * turns));
  Row cur, next;
  if (first < M) read(first + sub % PER, cur);
  Affine<LANES, CH> post, pre;
  post.load(a.post_gamma, a.post_beta, a.gate, lane, chunks);
  if (norm) pre.load(a.pre_gamma, a.pre_beta, nullptr, lane, chunks);
  for (int64_t m0 = first; m0 < end; m0 += step) {
    const int64_t m = m0 + sub % PER;
    const bool store = m < M;
    if (m0 + step < end) read(m + step, next);
    float v[CH][8], f[8];
    uint4 y[CH];
#pragma unroll
    for (int j = 0; j < CH; ++j) unpack8(cur.b[j], v[j]);
    if (a.post_gamma) normalise<LANES, CH, RMS>(v, lane, chunks, inv_d, a.eps, lds, turn);
#pragma unroll
    for (int j = 0; j < CH; ++j) {
      const int c = j * LANES + lane;
      const bool in = c < chunks;
#pragma unroll
      for (int i = 0; i < 8; ++i) v[j][i] = in ? fmaf(v[j][i], post.g[j][i], post.b[j][i]) : 0.0f;
      if (a.gate_rows) {
        unpack8(cur.g[j], f);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[j][i] *= f[i];
      }
      unpack8(cur.x[j], f);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[j][i] = fmaf(a.res_scale, f[i], v[j][i]);
      y[j] = pack8(v[j]);
    }
    if (norm) {
      // The next block's norm reads the stream before its rounding to bf16.
      normalise<LANES, CH, RMS>(v, lane, chunks, inv_d, a.eps, lds, turn);
#pragma unroll
      for (int j = 0; j < CH; ++j) {
        const bool in = j * LANES + lane < chunks;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[j][i] = in ? fmaf(v[j][i], pre.g[j][i], pre.b[j][i]) : 0.0f;
      }
    }
#pragma unroll
    for (int j = 0; j < CH; ++j) {
      const int c = j * LANES + lane;
      if (store && c < chunks) {
        if (a.y) store16(a.y + m * a.ld_y + 8 * c, y[j]);
        if (a.z) store16(a.z + m * a.ld_z + 8 * c, pack8(v[j]));
      }
    }
    if (a.zq)
      store_quantized<LANES, CH>(
          [&](int j, float* t) {
#pragma unroll
            for (int i = 0; i < 8; ++i) t[i] = v[j][i];
          },
          lane, (d + 127) / 128 * 16, store, a.zq + m * a.ld_zq, a.zq_scale + m, lds, turn);
    cur = next;
  }
}

}  // namespace

static int64_t groups(int64_t M, int lanes) {
  const int rows = block_of(lanes) / lanes;
  return (M + rows - 1) / rows;
}

// Most workgroups of a launch: a grid's threads are a 32-bit number.
constexpr int64_t MOST_GROUPS = 1 << 22;

// Lanes and chunks that hold a padded row: as few features a lane as fill a
// wave (rows of up to 256 share one), and a workgroup beyond 1024.
hipError_t launch_quantize_rows(int64_t M, int K, const uint16_t* x, int64_t ld_x, int8_t* q,
                                int64_t ld_q, float* scale, hipStream_t stream) {
  if (M <= 0) return hipSuccess;
  const int n = (int)i8_columns(K) / 8;
#define SURGE_LAUNCH(LANES, CH)                                                         \
  hipLaunchKernelGGL((quantize_rows_kernel<LANES, CH>), dim3((unsigned)std::min(groups(M, LANES), MOST_GROUPS)), \
                     dim3(block_of(LANES)), 0, stream, M, K, x, ld_x, q, ld_q, scale)
  if (n <= 32)
    SURGE_LAUNCH(16, 2);
  else if (n <= 64)
    SURGE_LAUNCH(32, 2);
  else if (n <= 256)
    SURGE_LAUNCH(64, 4);
  else if (n <= 1024)
    SURGE_LAUNCH(256, 4);
  else
    SURGE_LAUNCH(256, 8);
#undef SURGE_LAUNCH
  return hipGetLastError();
}

// Turns: as many as let one round of three workgroups per CU take all rows, so
// that no few workgroups are left for a second one (13,579 rows of 768: 20.3
// us, with 4 turns 23.6), and 4 where the rounds are many (200,003 rows of
// 1024 with gate rows, turns 1 / 2 / 4 / 8: 345 / 341 / 341 / 369; of 768 with
// a gate 304 / 242 / 227 / 232).  Rows beyond 4096 in 512 lanes of two chunks:
// 20,000 of 8192 306 us, in 256 of four 323, in 1024 of one 328.
hipError_t launch_block_norm(int64_t M, int d, bool rms, const BlockNorm& a, int n_cus,
                             hipStream_t stream) {
  if (M <= 0) return hipSuccess;
  const int n = (int)i8_columns(d) / 8;
#define SURGE_LAUNCH_KIND(LANES, CH, RMS)                                                      \
  {                                                                                            \
    const int64_t n_groups = groups(M, LANES);                                                 \
    const int64_t turns = n_groups > 18 * n_cus                                                \
                              ? std::max<int64_t>(4, (n_groups + MOST_GROUPS - 1) / MOST_GROUPS) \
                              : (n_groups + 3 * n_cus - 1) / (3 * n_cus);                      \
    hipLaunchKernelGGL((block_norm_kernel<LANES, CH, RMS>),                                    \
                       dim3((unsigned)((n_groups + turns - 1) / turns)), dim3(block_of(LANES)), 0, \
                       stream, M, d, (int)turns, a);                                           \
  }
#define SURGE_LAUNCH(LANES, CH)        \
  if (rms)                             \
    SURGE_LAUNCH_KIND(LANES, CH, true) \
  else                                 \
    SURGE_LAUNCH_KIND(LANES, CH, false)
  if (n <= 16) {
    SURGE_LAUNCH(16, 1);
  } else if (n <= 32) {
    SURGE_LAUNCH(32, 1);
  } else if (n <= 64) {
    SURGE_LAUNCH(64, 1);
  } else if (n <= 128) {
    SURGE_LAUNCH(64, 2);
  } else if (n <= 256) {
    SURGE_LAUNCH(256, 1);
  } else if (n <= 512) {
    SURGE_LAUNCH(256, 2);
  } else {
    SURGE_LAUNCH(512, 2);
  }
#undef SURGE_LAUNCH
#undef SURGE_LAUNCH_KIND
  return hipGetLastError();
}

}  // namespace surge
