// Host-side launchers of the operators of models that read the encoder's
// token states.  As in kernels.h the caller has checked the arguments.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace surge {

// Columns of the int8 rows that the quantizing kernels write: the features,
// padded with zeros to whole 128-byte stages of the int8 linear layer.
inline int64_t i8_columns(int64_t k) { return (k + 127) / 128 * 128; }

// q[m][k] = rne(x[m][k] * (127 / a)), scale[m] = a / 127 with
// a = max(max_k |x[m][k]|, 2^-100); columns K .. i8_columns(K) of q are 0.  A
// row with a value that is not finite gets q = 0 and scale = NaN.
// K % 8 == 0, K <= QUANTIZE_MAX_K.
constexpr int QUANTIZE_MAX_K = 16384;
hipError_t launch_quantize_rows(int64_t M, int K, const uint16_t* x, int64_t ld_x, int8_t* q,
                                int64_t ld_q, float* scale, hipStream_t stream);

// y = res_scale x + gate gate_rows N(block), z = N'(y), see
// surge_op_block_norm.  d % 8 == 0, d <= BLOCK_NORM_MAX_D.
constexpr int BLOCK_NORM_MAX_D = 8192;
struct BlockNorm {
  const uint16_t *x, *block, *gate_rows;  // block, gate_rows: NULL for none
  int64_t ld_x, ld_block, ld_gate;
  const float *post_gamma, *post_beta;    // post_gamma NULL: no norm; beta NULL: none
  const float* gate;                      // [d] or NULL
  const float *pre_gamma, *pre_beta;
  float res_scale, eps;
  uint16_t *y, *z;                        // NULL: not stored
  int64_t ld_y, ld_z;
  int8_t* zq;                             // z as int8 rows, NULL: not stored
  int64_t ld_zq;
  float* zq_scale;
};
hipError_t launch_block_norm(int64_t M, int d, bool rms, const BlockNorm& a, int n_cus,
                             hipStream_t stream);

// y[m][n] = epi(x_scale[m] w_scale[n] sum_k x[m][k] w[n][k] + bias[n]), epi 0
// nothing, 1 GELU, 2 + res[m][n].  K % 128 == 0, N % 8 == 0.
struct LinearI8 {
  const int8_t *x, *w;
  int64_t ld_x;
  const float *x_scale, *w_scale, *bias;
  const uint16_t* res;
  int64_t ld_res;
  uint16_t* y;
  int64_t ld_y;
};
hipError_t launch_linear_i8(int64_t M, int N, int K, int epi, const LinearI8& a, int n_cus,
                            hipStream_t stream);
// The tile of its first (or only) launch, rows << 16 | channels.
int linear_i8_tile(int64_t M, int N, int K, int n_cus);

}  // namespace surge
