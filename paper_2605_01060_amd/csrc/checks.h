// Argument checks shared by the asynchronous operators' entry points.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <atomic>

#include "internal.h"
#include "kernels.h"

#define HIP_TRY(expr)                                                                     \
  do {                                                                                    \
    hipError_t e_ = (expr);                                                               \
    if (e_ != hipSuccess)                                                                 \
      return fail(e_ == hipErrorOutOfMemory ? SURGE_ERR_OUT_OF_MEMORY : SURGE_ERR_DEVICE, \
                  "%s failed: %s", #expr, hipGetErrorString(e_));                         \
  } while (0)

#define CHECK(expr)                     \
  do {                                  \
    const surge_status st_ = (expr);    \
    if (st_ != SURGE_OK) return st_;    \
  } while (0)

namespace surge {

// Row strides are bounded so that the offset of a row within a tile or key
// block fits 32 bits.
constexpr int64_t kMaxStride = 1 << 22;

inline bool aligned(const void* p, uintptr_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

// A matrix of `rows` x `cols` elements, `ld` apart, read or written 16 bytes
// at a time.
inline surge_status check_matrix(const char* name, const void* p, int64_t cols, int64_t ld, int unit) {
  if (!p) return fail(SURGE_ERR_INVALID_ARGUMENT, "%s is NULL", name);
  if (!aligned(p, 16)) return fail(SURGE_ERR_INVALID_ARGUMENT, "%s must be 16-byte aligned", name);
  if (ld < cols || ld > kMaxStride || ld % unit)
    return fail(SURGE_ERR_INVALID_ARGUMENT,
                "row stride %lld of %s: a multiple of %d in [%lld, %lld] is needed", (long long)ld,
                name, unit, (long long)cols, (long long)kMaxStride);
  return SURGE_OK;
}

inline surge_status check_vector(const char* name, const void* p, bool needed) {
  if (!p && needed) return fail(SURGE_ERR_INVALID_ARGUMENT, "%s is NULL", name);
  if (!aligned(p, 16)) return fail(SURGE_ERR_INVALID_ARGUMENT, "%s must be 16-byte aligned", name);
  return SURGE_OK;
}

// An output in the place of an input (`over` says whether it may be, with the
// same stride) or of another output.
inline surge_status check_place(const char* name, const void* p, int64_t ld, const char* other, const void* q,
                         int64_t ld_other, bool over) {
  if (!p || p != q || (over && ld == ld_other)) return SURGE_OK;
  return fail(SURGE_ERR_INVALID_ARGUMENT, over ? "%s over %s needs its stride" : "%s is %s", name, other);
}

inline surge_status check_rows(int64_t M) {
  if (M < 0 || M > (int64_t)INT32_MAX)
    return fail(SURGE_ERR_INVALID_ARGUMENT, "M=%lld outside [0, 2^31)", (long long)M);
  return SURGE_OK;
}

// The current device and its compute units, asked for once a device, and that
// the stream is one of this device's.
inline surge_status current_device(hipStream_t stream, int* dev, int* n_cus) {
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

}  // namespace surge
