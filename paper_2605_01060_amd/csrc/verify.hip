// The check of drafted tokens against a target's probabilities (gfx950), see
// surge_op_verify_drafts.
//
// A sequence is a workgroup.  Its drafts are looked at together; then the one
// row of probabilities that decides the next token is summed in parts of 4096
// tokens, and the part in which the sum passes u times the whole is scanned
// again.  Sums are in 64 bits: in 32, u near a border of two tokens would take
// the wrong one in one of 10^5 calls or so of a large vocabulary.
#include "cache_device.h"

namespace surge {
namespace {

constexpr int WAVES = 16, PART = 4096, PER = PART / (64 * WAVES);
constexpr int MAX_PARTS = 1024;  // of a row: a vocabulary of 2^22

__device__ __forceinline__ double wave_sum64(double v) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

// The drafts of a sequence that are accepted, looked at by a wave: the first
// that is not ends them.
__device__ __forceinline__ int accepted_drafts(const VerifyDrafts& a, int64_t seq, int n) {
  const int lane = threadIdx.x & 63;
  for (int j0 = 0; j0 < n; j0 += 64) {
    const int j = j0 + lane;
    bool ok = false;
    if (j < n) {
      const int x = a.drafts[seq * a.max_drafts + j];
      if (x >= 0 && x < a.vocab) {
        const double p = a.p[(seq * (a.max_drafts + 1) + j) * a.ld_p + x];
        const double q = a.q ? (double)a.q[(seq * a.max_drafts + j) * a.ld_q + x] : 1.0;
        ok = (double)a.u[seq * (a.max_drafts + 1) + j] * q < p;
      }
    }
    const uint64_t failed = ~__ballot(ok);
    if (failed) return min(n, j0 + __builtin_ctzll(failed));
  }
  return n;
}

// What token v weighs: max(p - q, 0), without q all of p but for the draft;
// not above 0 (NaN too) is 0.
struct Weights {
  const float *p, *q;
  int without;
  __device__ __forceinline__ double operator()(int v) const {
    double d = p[v];
    if (q) d -= (double)q[v];
    return d > 0.0 && v != without ? d : 0.0;
  }
};

__global__ __launch_bounds__(64 * WAVES) void verify_kernel(VerifyDrafts a) {
  __shared__ double parts[MAX_PARTS], wave_sums[WAVES];
  __shared__ int shared_int[2];
  const int64_t seq = blockIdx.x;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int n = a.n_drafts ? min(max(a.n_drafts[seq], 0), a.max_drafts) : a.max_drafts;
  const int acc = accepted_drafts(a, seq, n);
  Weights w;
  w.p = a.p + (seq * (a.max_drafts + 1) + acc) * a.ld_p;
  w.q = acc < n && a.q ? a.q + (seq * a.max_drafts + acc) * a.ld_q : nullptr;
  w.without = acc < n && !a.q ? a.drafts[seq * a.max_drafts + acc] : -1;
  const int n_parts = (a.vocab + PART - 1) / PART;

  double total = 0.0;
  for (int attempt = 0; attempt < 2; ++attempt) {
    // A wave sums whole parts.
    for (int part = wave; part < n_parts; part += WAVES) {
      double s = 0.0;
#pragma unroll 8
      for (int i = 0; i < PART / 64; ++i) {
        const int v = part * PART + i * 64 + lane;
        if (v < a.vocab) s += w(v);
      }
      s = wave_sum64(s);
      if (lane == 0) parts[part] = s;
    }
    __syncthreads();
    total = 0.0;
    for (int i = 0; i < n_parts; ++i) total += parts[i];
    __syncthreads();
    // Nothing left over by q: the target's own probabilities.
    if (total > 0.0 || (!w.q && w.without < 0)) break;
    w.q = nullptr;
    w.without = -1;
  }
  int token = -1;
  if (total > 0.0 && total < HUGE_VAL) {
    const double target = (double)a.u[seq * (a.max_drafts + 1) + a.max_drafts] * total;
    // The part in which the sum passes the target, else the last one that
    // weighs anything.
    int part = 0;
    double before = 0.0, sum = 0.0;
    for (int i = 0; i < n_parts; ++i) {
      const double s = parts[i];
      if (s > 0.0) {
        part = i;
        before = sum;
        if (sum + s > target) break;
      }
      sum += s;
    }
    // A thread's PER tokens, a wave's, the part's.
    double mine[PER], s = 0.0;
    const int v0 = part * PART + (int)threadIdx.x * PER;
    int last = -1;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      mine[i] = v0 + i < a.vocab ? w(v0 + i) : 0.0;
      s += mine[i];
      if (mine[i] > 0.0) last = v0 + i;
    }
    double upto = s;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const double x = __shfl_up(upto, o, 64);
      if (lane >= o) upto += x;
    }
    if (lane == 63) wave_sums[wave] = upto;
    if (threadIdx.x == 0) {
      shared_int[0] = INT32_MAX;  // the first token beyond the target
      shared_int[1] = -1;         // the last one that weighs anything
    }
    __syncthreads();
    double c = before + (upto - s);
    for (int i = 0; i < wave; ++i) c += wave_sums[i];
    int first = INT32_MAX;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      c += mine[i];
      if (first == INT32_MAX && mine[i] > 0.0 && c > target) first = v0 + i;
    }
    if (first != INT32_MAX) atomicMin(&shared_int[0], first);
    if (last >= 0) atomicMax(&shared_int[1], last);
    __syncthreads();
    token = shared_int[0] != INT32_MAX ? shared_int[0] : shared_int[1];
  }
  for (int j = threadIdx.x; j <= a.max_drafts; j += 64 * WAVES)
    a.tokens[seq * (a.max_drafts + 1) + j] = j < acc ? a.drafts[seq * a.max_drafts + j] : j == acc ? token : -1;
  if (threadIdx.x == 0) a.accepted[seq] = acc;
}

}  // namespace

hipError_t launch_verify_drafts(int64_t n_seqs, const VerifyDrafts& a, hipStream_t stream) {
  hipLaunchKernelGGL(verify_kernel, dim3((unsigned)n_seqs), dim3(64 * WAVES), 0, stream, a);
  return hipGetLastError();
}

}  // namespace surge
