// Entry points of the operators of models that read the encoder's token
// states: argument checks, the cross-attention plan and the launches.
#include <math.h>

#include <algorithm>
#include <atomic>
#include <exception>
#include <new>

#include "cross.h"
#include "internal.h"
#include "kernels.h"
#include "reader.h"
#include "surge_ops.h"

using namespace surge;

#define HIP_TRY(expr)                                                                     \
  do {                                                                                    \
    hipError_t e_ = (expr);                                                               \
    if (e_ != hipSuccess)                                                                 \
      return fail(e_ == hipErrorOutOfMemory ? SURGE_ERR_OUT_OF_MEMORY : SURGE_ERR_DEVICE, \
                  "%s failed: %s", #expr, hipGetErrorString(e_));                         \
  } while (0)

struct surge_cross_plan {
  int device = 0;
  int n_kv_heads = 0, group = 0, d_head = 0;
  int64_t q_tokens = 0, kv_tokens = 0;
  int n_items[CROSS_CLASSES] = {}, n_units = 0, n_joins = 0, max_parts = 0;
  int64_t n_parts = 0;   // slots of 32 rows in the workspace
  int n_split = 0;       // of the units, those that hold a part of their rows' keys
  bool short_blocks = false;
  void* lists = nullptr;  // device: the items of each class, then the joins
};

namespace {

// Row strides are bounded so that the offset of a row within a tile or key
// block fits 32 bits.
constexpr int64_t kMaxStride = 1 << 22;

bool aligned(const void* p, uintptr_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

// A matrix of `rows` x `cols` elements, `ld` apart, read or written 16 bytes
// at a time.
surge_status check_matrix(const char* name, const void* p, int64_t cols, int64_t ld, int unit) {
  if (!p) return fail(SURGE_ERR_INVALID_ARGUMENT, "%s is NULL", name);
  if (!aligned(p, 16)) return fail(SURGE_ERR_INVALID_ARGUMENT, "%s must be 16-byte aligned", name);
  if (ld < cols || ld > kMaxStride || ld % unit)
    return fail(SURGE_ERR_INVALID_ARGUMENT,
                "row stride %lld of %s: a multiple of %d in [%lld, %lld] is needed", (long long)ld,
                name, unit, (long long)cols, (long long)kMaxStride);
  return SURGE_OK;
}

surge_status check_vector(const char* name, const void* p, bool needed) {
  if (!p && needed) return fail(SURGE_ERR_INVALID_ARGUMENT, "%s is NULL", name);
  if (!aligned(p, 16)) return fail(SURGE_ERR_INVALID_ARGUMENT, "%s must be 16-byte aligned", name);
  return SURGE_OK;
}

// An output in the place of an input (`over` says whether it may be, with the
// same stride) or of another output.
surge_status check_place(const char* name, const void* p, int64_t ld, const char* other, const void* q,
                         int64_t ld_other, bool over) {
  if (!p || p != q || (over && ld == ld_other)) return SURGE_OK;
  return fail(SURGE_ERR_INVALID_ARGUMENT, over ? "%s over %s needs its stride" : "%s is %s", name, other);
}

surge_status check_rows(int64_t M) {
  if (M < 0 || M > (int64_t)INT32_MAX)
    return fail(SURGE_ERR_INVALID_ARGUMENT, "M=%lld outside [0, 2^31)", (long long)M);
  return SURGE_OK;
}

// Rows of queries and of keys are counted in 32 bits, a block of them beyond
// the last one too.
constexpr int64_t kMostRows = INT32_MAX - 255;

// cu[0] = 0, never decreasing, at most kMostRows.
surge_status check_offsets(const char* name, int64_t n, const int64_t* cu) {
  if (!cu) return fail(SURGE_ERR_INVALID_ARGUMENT, "%s is NULL", name);
  if (cu[0] != 0) return fail(SURGE_ERR_INVALID_ARGUMENT, "%s[0] != 0", name);
  for (int64_t i = 0; i < n; ++i)
    if (cu[i + 1] < cu[i])
      return fail(SURGE_ERR_INVALID_ARGUMENT, "%s decreases at %lld", name, (long long)i);
  if (cu[n] > kMostRows) return fail(SURGE_ERR_INVALID_ARGUMENT, "%s: too many rows", name);
  return SURGE_OK;
}

// The current device and its compute units, asked for once a device, and that
// the stream is one of this device's.
surge_status current_device(hipStream_t stream, int* dev, int* n_cus) {
  constexpr int kMaxDevices = 64;
  static std::atomic<int> known[kMaxDevices];
  HIP_TRY(hipGetDevice(dev));
  if (stream) {
    int own = 0;
    HIP_TRY(hipStreamGetDevice(stream, &own));
    if (own != *dev)
      return fail(SURGE_ERR_INVALID_ARGUMENT, "a stream of device %d, the current one is %d", own, *dev);
  }
  if (*dev < 0 || *dev >= kMaxDevices)
    return fail(SURGE_ERR_DEVICE, "device index %d outside [0, %d)", *dev, kMaxDevices);
  *n_cus = known[*dev].load(std::memory_order_relaxed);
  if (*n_cus > 0) return SURGE_OK;
  HIP_TRY(resolve_cus(n_cus));
  known[*dev].store(*n_cus, std::memory_order_relaxed);
  return SURGE_OK;
}

#define CHECK(expr)                     \
  do {                                  \
    const surge_status st_ = (expr);    \
    if (st_ != SURGE_OK) return st_;    \
  } while (0)

int64_t part_rows(const surge_cross_plan* p) { return p->n_parts * p->n_kv_heads * 32; }
int64_t workspace_bytes(const surge_cross_plan* p) {
  return part_rows(p) * (8 + 4 * (int64_t)p->d_head);
}

}  // namespace

extern "C" {

surge_status surge_op_quantize_rows(int64_t M, int32_t K, const uint16_t* d_x, int64_t ld_x,
                                    int8_t* d_q, int64_t ld_q, float* d_scale, void* hip_stream) {
  clear_error();
  CHECK(check_rows(M));
  if (K < 8 || K > QUANTIZE_MAX_K || K % 8)
    return fail(SURGE_ERR_INVALID_ARGUMENT, "K=%d: a multiple of 8 in [8, %d] is needed", K,
                QUANTIZE_MAX_K);
  if (M == 0) return SURGE_OK;
  CHECK(check_matrix("x", d_x, K, ld_x, 8));
  CHECK(check_matrix("q", d_q, i8_columns(K), ld_q, 16));
  if (!d_scale) return fail(SURGE_ERR_INVALID_ARGUMENT, "scale is NULL");
  CHECK(check_place("q", d_q, 0, "x", d_x, 0, false));
  int dev = 0, n_cus = 0;
  CHECK(current_device((hipStream_t)hip_stream, &dev, &n_cus));
  HIP_TRY(launch_quantize_rows(M, K, d_x, ld_x, d_q, ld_q, d_scale, (hipStream_t)hip_stream));
  return SURGE_OK;
}

surge_status surge_op_linear_i8(int64_t M, int32_t N, int32_t K, const int8_t* d_x, int64_t ld_x,
                                const float* d_x_scale, const int8_t* d_w, const float* d_w_scale,
                                const float* d_bias, const uint16_t* d_res, int64_t ld_res,
                                int32_t epilogue, uint16_t* d_y, int64_t ld_y, void* hip_stream) {
  clear_error();
  CHECK(check_rows(M));
  if (N < 8 || N % 8 || N > 1 << 20)
    return fail(SURGE_ERR_INVALID_ARGUMENT, "N=%d: a multiple of 8 in [8, 2^20] is needed", N);
  if (K < 128 || K % 128 || K > 65536)
    return fail(SURGE_ERR_INVALID_ARGUMENT, "K=%d: a multiple of 128 in [128, 65536] is needed", K);
  if (epilogue < 0 || epilogue > 2)
    return fail(SURGE_ERR_INVALID_ARGUMENT, "epilogue=%d", epilogue);
  if (M == 0) return SURGE_OK;
  CHECK(check_matrix("x", d_x, K, ld_x, 16));
  CHECK(check_matrix("y", d_y, N, ld_y, 8));
  if (epilogue == 2) CHECK(check_matrix("res", d_res, N, ld_res, 8));
  if (!d_x_scale) return fail(SURGE_ERR_INVALID_ARGUMENT, "x_scale is NULL");
  CHECK(check_vector("w", d_w, true));
  CHECK(check_vector("w_scale", d_w_scale, true));
  CHECK(check_vector("bias", d_bias, true));
  CHECK(check_place("y", d_y, 0, "x", d_x, 0, false));
  CHECK(check_place("y", d_y, 0, "w", d_w, 0, false));
  if (epilogue == 2) CHECK(check_place("y", d_y, ld_y, "res", d_res, ld_res, true));
  int dev = 0, n_cus = 0;
  CHECK(current_device((hipStream_t)hip_stream, &dev, &n_cus));
  const LinearI8 a = {d_x,    d_w,    ld_x, d_x_scale, d_w_scale, d_bias,
                      d_res, ld_res, d_y,  ld_y};
  HIP_TRY(launch_linear_i8(M, N, K, epilogue, a, n_cus, (hipStream_t)hip_stream));
  return SURGE_OK;
}

int32_t surge_op_linear_i8_tile(int64_t M, int32_t N, int32_t K, int32_t n_cus) {
  if (M < 1 || M > (int64_t)INT32_MAX || N < 8 || N % 8 || N > 1 << 20 || K < 128 || K % 128 ||
      K > 65536 || n_cus < 1)
    return 0;
  return linear_i8_tile(M, N, K, n_cus);
}

surge_status surge_op_block_norm(int64_t M, int32_t d, int32_t kind, const uint16_t* d_x,
                                 int64_t ld_x, const uint16_t* d_block, int64_t ld_block,
                                 const float* d_post_gamma, const float* d_post_beta,
                                 const float* d_gate, const uint16_t* d_gate_rows, int64_t ld_gate,
                                 float res_scale, const float* d_pre_gamma, const float* d_pre_beta,
                                 float eps, uint16_t* d_y, int64_t ld_y, uint16_t* d_z, int64_t ld_z,
                                 int8_t* d_zq, int64_t ld_zq, float* d_zq_scale, void* hip_stream) {
  clear_error();
  CHECK(check_rows(M));
  if (d < 8 || d > BLOCK_NORM_MAX_D || d % 8)
    return fail(SURGE_ERR_INVALID_ARGUMENT, "d=%d: a multiple of 8 in [8, %d] is needed", d,
                BLOCK_NORM_MAX_D);
  if (kind != SURGE_NORM_LAYER && kind != SURGE_NORM_RMS)
    return fail(SURGE_ERR_INVALID_ARGUMENT, "kind=%d", kind);
  if (!isfinite(res_scale)) return fail(SURGE_ERR_INVALID_ARGUMENT, "res_scale is not finite");
  if (!d_block && (d_post_gamma || d_gate || d_gate_rows))
    return fail(SURGE_ERR_INVALID_ARGUMENT, "post norm or gate without a block output");
  const bool norm = d_z || d_zq;
  if (!norm && !d_y) return fail(SURGE_ERR_INVALID_ARGUMENT, "no output");
  if ((norm || d_post_gamma) && !(eps >= 0.0f && eps <= 1.0f))
    return fail(SURGE_ERR_INVALID_ARGUMENT, "eps=%g outside [0, 1]", (double)eps);
  if (d_post_beta && (!d_post_gamma || kind == SURGE_NORM_RMS))
    return fail(SURGE_ERR_INVALID_ARGUMENT, "post_beta without a LayerNorm after the block");
  if (d_pre_beta && (!norm || kind == SURGE_NORM_RMS))
    return fail(SURGE_ERR_INVALID_ARGUMENT, "pre_beta without a LayerNorm before the next block");
  if (M == 0) return SURGE_OK;
  CHECK(check_matrix("x", d_x, d, ld_x, 8));
  if (d_block) CHECK(check_matrix("block", d_block, d, ld_block, 8));
  if (d_gate_rows) CHECK(check_matrix("gate_rows", d_gate_rows, d, ld_gate, 8));
  if (d_y) CHECK(check_matrix("y", d_y, d, ld_y, 8));
  if (d_z) CHECK(check_matrix("z", d_z, d, ld_z, 8));
  if (d_zq) {
    CHECK(check_matrix("zq", d_zq, i8_columns(d), ld_zq, 16));
    if (!d_zq_scale) return fail(SURGE_ERR_INVALID_ARGUMENT, "zq_scale is NULL");
  }
  CHECK(check_vector("post_gamma", d_post_gamma, false));
  CHECK(check_vector("post_beta", d_post_beta, false));
  CHECK(check_vector("gate", d_gate, false));
  CHECK(check_vector("pre_gamma", d_pre_gamma, norm));
  CHECK(check_vector("pre_beta", d_pre_beta, false));
  const struct {
    const char* name;
    const void* p;
    int64_t ld;
  } ins[] = {{"x", d_x, ld_x}, {"block", d_block, ld_block}, {"gate_rows", d_gate_rows, ld_gate}};
  for (const auto& in : ins) {
    CHECK(check_place("y", d_y, ld_y, in.name, in.p, in.ld, true));
    CHECK(check_place("z", d_z, ld_z, in.name, in.p, in.ld, true));
    CHECK(check_place("zq", d_zq, 0, in.name, in.p, 0, false));
  }
  CHECK(check_place("z", d_z, 0, "y", d_y, 0, false));
  CHECK(check_place("zq", d_zq, 0, "y", d_y, 0, false));
  CHECK(check_place("zq", d_zq, 0, "z", d_z, 0, false));
  const BlockNorm a = {d_x,         d_block,    d_gate_rows, ld_x, ld_block, ld_gate, d_post_gamma,
                       d_post_beta, d_gate,     d_pre_gamma, d_pre_beta, res_scale, eps, d_y, d_z,
                       ld_y,        ld_z,       d_zq,        ld_zq, d_zq_scale};
  int dev = 0, n_cus = 0;
  CHECK(current_device((hipStream_t)hip_stream, &dev, &n_cus));
  HIP_TRY(launch_block_norm(M, d, kind == SURGE_NORM_RMS, a, n_cus, (hipStream_t)hip_stream));
  return SURGE_OK;
}

surge_status surge_cross_plan_create(int64_t n_seqs, const int64_t* h_cu_q, const int64_t* h_cu_kv,
                                     int32_t n_heads, int32_t n_kv_heads, int32_t d_head,
                                     surge_cross_plan** out) {
  clear_error();
  if (!out) return fail(SURGE_ERR_INVALID_ARGUMENT, "out is NULL");
  *out = nullptr;
  if (n_seqs < 1 || n_seqs > (int64_t)INT32_MAX)
    return fail(SURGE_ERR_INVALID_ARGUMENT, "n_seqs=%lld", (long long)n_seqs);
  if (d_head != 32 && d_head != 64 && d_head != 128)
    return fail(SURGE_ERR_INVALID_ARGUMENT, "d_head=%d", d_head);
  if (n_heads < 1 || n_heads > 1024 || n_kv_heads < 1 || n_heads % n_kv_heads)
    return fail(SURGE_ERR_INVALID_ARGUMENT, "n_heads=%d, n_kv_heads=%d", n_heads, n_kv_heads);
  CHECK(check_offsets("cu_q", n_seqs, h_cu_q));
  CHECK(check_offsets("cu_kv", n_seqs, h_cu_kv));
  const int group = n_heads / n_kv_heads;
  if (h_cu_q[n_seqs] * group > kMostRows)
    return fail(SURGE_ERR_CAPACITY, "too many rows of queries and heads");
  try {
    CrossList list;
    int dev = 0, n_cus = 0;
    CHECK(current_device(nullptr, &dev, &n_cus));
    build_cross_list(n_seqs, h_cu_q, h_cu_kv, n_kv_heads, group, d_head, n_cus, &list);
    // A launch's threads are a 32-bit number, two waves for each 32 rows of a
    // unit at most and sixteen for a joined row.
    int64_t items = 0;
    bool fits = (int64_t)list.joins.size() * n_kv_heads <= (1 << 16);
    for (int c = 0; c < CROSS_CLASSES; ++c) {
      items += (int64_t)list.items[c].size();
      fits = fits && (int64_t)list.items[c].size() * n_kv_heads * CROSS_ROWS[c] <= (int64_t)INT32_MAX;
    }
    if (!fits || items > (int64_t)INT32_MAX)
      return fail(SURGE_ERR_CAPACITY, "too many units of work for one plan");
    surge_cross_plan* p = new surge_cross_plan;
    p->n_kv_heads = n_kv_heads;
    p->group = group;
    p->d_head = d_head;
    p->q_tokens = h_cu_q[n_seqs];
    p->kv_tokens = h_cu_kv[n_seqs];
    for (int c = 0; c < CROSS_CLASSES; ++c) p->n_items[c] = (int)list.items[c].size();
    p->n_units = (int)items;
    for (const auto& v : list.items)
      for (const CrossItem& it : v) p->n_split += it.part >= 0;
    p->n_joins = (int)list.joins.size();
    p->max_parts = list.max_parts;
    p->n_parts = list.n_parts;
    p->short_blocks = list.short_blocks;
    const size_t bytes = items * sizeof(CrossItem) + list.joins.size() * sizeof(CrossJoin);
    p->device = dev;
    hipError_t e = hipSuccess;
    if (bytes > 0) e = hipMalloc(&p->lists, bytes);
    char* at = (char*)p->lists;
    auto upload = [&](const void* from, size_t n) {
      if (e == hipSuccess && n > 0) e = hipMemcpy(at, from, n, hipMemcpyHostToDevice);
      at += n;
    };
    for (const auto& v : list.items) upload(v.data(), v.size() * sizeof(CrossItem));
    upload(list.joins.data(), list.joins.size() * sizeof(CrossJoin));
    if (e != hipSuccess) {
      surge_cross_plan_destroy(p);
      return fail(e == hipErrorOutOfMemory ? SURGE_ERR_OUT_OF_MEMORY : SURGE_ERR_DEVICE,
                  "the plan's lists: %s", hipGetErrorString(e));
    }
    *out = p;
  } catch (const std::bad_alloc&) {
    return fail(SURGE_ERR_OUT_OF_MEMORY, "host memory for the plan");
  } catch (const std::exception& e) {
    return fail(SURGE_ERR_INTERNAL, "the plan's list: %s", e.what());
  }
  return SURGE_OK;
}

void surge_cross_plan_destroy(surge_cross_plan* plan) {
  if (!plan) return;
  if (plan->lists) {
    int dev = 0;
    const bool moved = hipGetDevice(&dev) == hipSuccess && dev != plan->device &&
                       hipSetDevice(plan->device) == hipSuccess;
    (void)hipFree(plan->lists);
    if (moved) (void)hipSetDevice(dev);
  }
  delete plan;
}

surge_status surge_cross_plan_info(const surge_cross_plan* plan, int64_t* bytes, int64_t* n_units,
                                   int64_t* n_parts) {
  clear_error();
  if (!plan) return fail(SURGE_ERR_INVALID_ARGUMENT, "plan is NULL");
  if (bytes) *bytes = workspace_bytes(plan);
  if (n_units) *n_units = (int64_t)plan->n_units * plan->n_kv_heads;
  if (n_parts) *n_parts = (int64_t)plan->n_split * plan->n_kv_heads;
  return SURGE_OK;
}

surge_status surge_op_cross_attention(const surge_cross_plan* plan, const uint16_t* d_q, int64_t ld_q,
                                      const uint16_t* d_k, int64_t ld_k, const uint16_t* d_v,
                                      int64_t ld_v, const uint8_t* d_key_mask, float scale,
                                      void* d_workspace, int64_t n_workspace, uint16_t* d_out,
                                      int64_t ld_out, void* hip_stream) {
  clear_error();
  if (!plan) return fail(SURGE_ERR_INVALID_ARGUMENT, "plan is NULL");
  // Times log2(e) it is still a float.
  const float scale_log2 = scale * 1.4426950408889634f;
  if (!(scale > 0.0f) || !isfinite(scale_log2))
    return fail(SURGE_ERR_INVALID_ARGUMENT, "scale=%g must be positive and below 2^127", (double)scale);
  if (plan->n_units == 0) return SURGE_OK;
  const int64_t kv_cols = (int64_t)plan->n_kv_heads * plan->d_head;
  const int64_t cols = kv_cols * plan->group;
  CHECK(check_matrix("q", d_q, cols, ld_q, 8));
  CHECK(check_matrix("out", d_out, cols, ld_out, 8));
  if (plan->kv_tokens > 0) {
    CHECK(check_matrix("k", d_k, kv_cols, ld_k, 8));
    CHECK(check_matrix("v", d_v, kv_cols, ld_v, 8));
  }
  if (d_out == d_q || d_out == d_k || d_out == d_v)
    return fail(SURGE_ERR_INVALID_ARGUMENT, "out is one of the inputs");
  const int64_t need = workspace_bytes(plan);
  if (need > 0) {
    CHECK(check_vector("workspace", d_workspace, true));
    if (n_workspace < need)
      return fail(SURGE_ERR_CAPACITY, "workspace of %lld bytes, %lld are needed",
                  (long long)n_workspace, (long long)need);
  }
  int dev = 0, n_cus = 0;
  CHECK(current_device((hipStream_t)hip_stream, &dev, &n_cus));
  if (dev != plan->device)
    return fail(SURGE_ERR_INVALID_ARGUMENT, "the plan was made on device %d, the current one is %d",
                plan->device, dev);
  CrossAttention a;
  a.q = d_q;
  a.k = d_k;
  a.v = d_v;
  a.ld_q = ld_q;
  a.ld_k = ld_k;
  a.ld_v = ld_v;
  a.mask = d_key_mask;
  a.scale_log2 = scale_log2;
  a.n_kv_heads = plan->n_kv_heads;
  a.group = plan->group;
  a.items = (const CrossItem*)plan->lists;
  std::copy(plan->n_items, plan->n_items + CROSS_CLASSES, a.n_items);
  a.joins = (const CrossJoin*)(a.items + plan->n_units);
  a.n_joins = plan->n_joins;
  a.max_parts = plan->max_parts;
  a.short_blocks = plan->short_blocks;
  a.part_o = (float*)d_workspace;
  a.part_ml = (float2*)((float*)d_workspace + part_rows(plan) * plan->d_head);
  a.out = d_out;
  a.ld_out = ld_out;
  HIP_TRY(launch_cross_attention(a, plan->d_head, (hipStream_t)hip_stream));
  return SURGE_OK;
}

}  // extern "C"
