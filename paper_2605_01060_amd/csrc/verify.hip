// The check of drafted tokens against a target's probabilities (gfx950), see
// surge_op_verify_drafts.
//
// The drafts of a sequence are looked at by one wave together; then the one row
// of probabilities that decides the next token is summed, in tiles of 4096
// tokens, and the tile in which the sum passes u times the whole is scanned.
// Sums are in 64 bits: in 32, u near a border of two tokens would take the wrong
// one in one of 10^3 calls or so of a large vocabulary.
//
// A workgroup of 16 waves holds eight tiles in registers, all of its loads in
// flight together.  A vocabulary of one workgroup's tiles is done in one launch;
// of a larger one a workgroup for each eight tiles leaves the tiles' sums, and a
// second launch chooses among them and reads the chosen tile again.
#include "cache_device.h"

namespace surge {
namespace {

constexpr int WAVES = 16, TILE = 64 * WAVES * 4, TILES = 8;
constexpr int MAX_TILES = (1 << 22) / TILE;  // of the largest vocabulary

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
    if (failed) return __builtin_amdgcn_readfirstlane(min(n, j0 + __builtin_ctzll(failed)));
  }
  return __builtin_amdgcn_readfirstlane(n);
}

// The row that the next token is drawn from: weights max(p - q, 0), without q
// all of p but for the draft; not above 0 (NaN too) is 0.  Rows are read through
// buffer descriptors of their length: they are 4-byte aligned, of any length,
// and what a load of four has beyond the end (each value is checked by itself), or
// in a row that is not there, is 0.
struct Row {
  __amdgpu_buffer_rsrc_t p, q;
  bool has_q;
  int without;
};

__device__ __forceinline__ __amdgpu_buffer_rsrc_t row_buffer(const float* row, int vocab) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(row), 0, row ? vocab * 4 : 0, 0x00027000);
}

__device__ __forceinline__ Row row_of(const VerifyDrafts& a, int64_t seq, int n, int acc) {
  Row r;
  r.has_q = acc < n && a.q;
  r.p = row_buffer(a.p + (seq * (a.max_drafts + 1) + acc) * a.ld_p, a.vocab);
  r.q = row_buffer(r.has_q ? a.q + (seq * a.max_drafts + acc) * a.ld_q : nullptr, a.vocab);
  r.without = acc < n && !a.q ? a.drafts[seq * a.max_drafts + acc] : -1;
  return r;
}

__device__ __forceinline__ f32x4 load4(__amdgpu_buffer_rsrc_t row, int v) {
  return __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(row, v * 4, 0, 0));
}

__device__ __forceinline__ int drafts_of(const VerifyDrafts& a, int64_t seq) {
  return a.n_drafts ? min(max(a.n_drafts[seq], 0), a.max_drafts) : a.max_drafts;
}

// The tokens v .. v + 3 of up to N tiles, v = first + i TILE + 4 thread.
template <int N>
struct Tokens {
  f32x4 p[N], q[N];
  __device__ __forceinline__ void load(const Row& r, int v) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      p[i] = load4(r.p, v + i * TILE);
      q[i] = load4(r.q, v + i * TILE);
    }
  }
  __device__ __forceinline__ double weight(const Row& r, int v, int i, int j) const {
    const double d = (double)p[i][j] - (double)q[i][j];
    return d > 0.0 && v + i * TILE + j != r.without ? d : 0.0;
  }
  __device__ __forceinline__ double sum(const Row& r, int v, int i) const {
    return (weight(r, v, i, 0) + weight(r, v, i, 1)) + (weight(r, v, i, 2) + weight(r, v, i, 3));
  }
};

// Sums of N tiles over the workgroup, in `shared`'s row WAVES for every thread.
template <int N>
__device__ __forceinline__ void tile_sums(double (*shared)[N], const double* s) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const double v = wave_sum64(s[i]);
    if (lane == 0) shared[wave][i] = v;
  }
  __syncthreads();
  if (threadIdx.x < N) {
    double v = 0.0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) v += shared[w][threadIdx.x];
    shared[WAVES][threadIdx.x] = v;
  }
  __syncthreads();
}

// The tile in which the sum of `n` tiles passes the target, else the last that
// weighs anything, and what the tiles before it weigh.
template <class Sum>
__device__ __forceinline__ int passing(Sum sum, int n, double target, double* before) {
  int tile = 0;
  double s = 0.0;
  *before = 0.0;
  for (int i = 0; i < n; ++i) {
    const double t = sum(i);
    if (t > 0.0) {
      tile = i;
      *before = s;
      if (s + t > target) break;
    }
    s += t;
  }
  return tile;
}

// The token of a tile, of which this thread's four weigh w, at which the sum
// passes the target, else the last that weighs anything.
__device__ __forceinline__ int token_of(const double* w, int v, double before, double target) {
  __shared__ double wave_sums[WAVES];
  __shared__ int found[2];  // the first token beyond the target, the last one that weighs anything
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const double s = (w[0] + w[1]) + (w[2] + w[3]);
  double upto = s;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const double x = __shfl_up(upto, o, 64);
    if (lane >= o) upto += x;
  }
  if (lane == 63) wave_sums[wave] = upto;
  if (threadIdx.x == 0) {
    found[0] = INT32_MAX;
    found[1] = -1;
  }
  __syncthreads();
  double c = before + (upto - s);
  for (int i = 0; i < wave; ++i) c += wave_sums[i];
  int first = INT32_MAX, last = -1;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    c += w[j];
    if (w[j] > 0.0) last = v + j;
    if (first == INT32_MAX && w[j] > 0.0 && c > target) first = v + j;
  }
  if (first != INT32_MAX) atomicMin(&found[0], first);
  if (last >= 0) atomicMax(&found[1], last);
  __syncthreads();
  return found[0] != INT32_MAX ? found[0] : found[1];
}

__device__ __forceinline__ bool drawable(double total) { return total > 0.0 && total < HUGE_VAL; }

__device__ __forceinline__ double target_of(const VerifyDrafts& a, int64_t seq, double total) {
  return (double)a.u[seq * (a.max_drafts + 1) + a.max_drafts] * total;
}

__device__ __forceinline__ void store_tokens(const VerifyDrafts& a, int64_t seq, int acc, int token) {
  for (int j = threadIdx.x; j <= a.max_drafts; j += 64 * WAVES)
    a.tokens[seq * (a.max_drafts + 1) + j] = j < acc ? a.drafts[seq * a.max_drafts + j] : j == acc ? token : -1;
  if (threadIdx.x == 0) a.accepted[seq] = acc;
}

// A vocabulary of at most N tiles: a workgroup a sequence, its row in registers.
template <int N>
__global__ __launch_bounds__(64 * WAVES) void verify_kernel(VerifyDrafts a) {
  __shared__ double shared[WAVES + 1][N];
  const int64_t seq = blockIdx.x;
  const int n = drafts_of(a, seq), acc = accepted_drafts(a, seq, n), v = (int)threadIdx.x * 4;
  Row r = row_of(a, seq, n, acc);
  Tokens<N> t;
  t.load(r, v);
  double s[N], total = 0.0;
  while (true) {
#pragma unroll
    for (int i = 0; i < N; ++i) s[i] = t.sum(r, v, i);
    tile_sums<N>(shared, s);
    total = 0.0;
#pragma unroll
    for (int i = 0; i < N; ++i) total += shared[WAVES][i];
    if (total > 0.0 || (!r.has_q && r.without < 0)) break;
    // Nothing left over by q: the target's own probabilities.
    r.has_q = false;
    r.without = -1;
#pragma unroll
    for (int i = 0; i < N; ++i) t.q[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    __syncthreads();  // the sums are read before they are made again
  }
  int token = -1;
  if (drawable(total)) {
    const double target = target_of(a, seq, total);
    double before, w[4];
    const int tile = passing([&](int i) { return shared[WAVES][i]; }, N, target, &before);
    Tokens<1> one = {{t.p[0]}, {t.q[0]}};
#pragma unroll
    for (int i = 1; i < N; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        one.p[0][j] = i == tile ? t.p[i][j] : one.p[0][j];
        one.q[0][j] = i == tile ? t.q[i][j] : one.q[0][j];
      }
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = one.weight(r, v + tile * TILE, 0, j);
    token = token_of(w, v + tile * TILE, before, target);
  }
  store_tokens(a, seq, acc, token);
}

// The tiles' sums of the row that decides, a workgroup for each TILES of them.
__global__ __launch_bounds__(64 * WAVES) void verify_sum_kernel(VerifyDrafts a, int groups, int tiles) {
  __shared__ double shared[WAVES + 1][TILES];
  const int64_t seq = blockIdx.x / groups;
  const int first = (int)(blockIdx.x % groups) * TILES;
  const int n = drafts_of(a, seq), acc = accepted_drafts(a, seq, n), v = first * TILE + (int)threadIdx.x * 4;
  const Row r = row_of(a, seq, n, acc);
  Tokens<TILES> t;
  t.load(r, v);
  double s[TILES];
#pragma unroll
  for (int i = 0; i < TILES; ++i) s[i] = t.sum(r, v, i);
  tile_sums<TILES>(shared, s);
  if (threadIdx.x < TILES && first + (int)threadIdx.x < tiles)
    a.sums[seq * tiles + first + threadIdx.x] = shared[WAVES][threadIdx.x];
}

__global__ __launch_bounds__(64 * WAVES) void verify_choose_kernel(VerifyDrafts a, int tiles) {
  __shared__ double sums[MAX_TILES];
  __shared__ double shared[WAVES + 1][1];
  const int64_t seq = blockIdx.x;
  const int n = drafts_of(a, seq), acc = accepted_drafts(a, seq, n);
  Row r = row_of(a, seq, n, acc);
  Tokens<1> t;
  double total = 0.0;
  for (int i = threadIdx.x; i < tiles; i += 64 * WAVES) sums[i] = a.sums[seq * tiles + i];
  __syncthreads();
  for (int i = 0; i < tiles; ++i) total += sums[i];
  if (!(total > 0.0) && (r.has_q || r.without >= 0)) {
    // Nothing left over by q: the target's own probabilities.
    r.q = row_buffer(nullptr, 0);
    r.without = -1;
    total = 0.0;
    for (int i = 0; i < tiles; ++i) {
      const int v = i * TILE + (int)threadIdx.x * 4;
      t.load(r, v);
      const double s = t.sum(r, v, 0);
      tile_sums<1>(shared, &s);
      if (threadIdx.x == 0) sums[i] = shared[WAVES][0];
      total += shared[WAVES][0];
      __syncthreads();
    }
    __syncthreads();
  }
  int token = -1;
  if (drawable(total)) {
    const double target = target_of(a, seq, total);
    double before, w[4];
    const int tile = passing([&](int i) { return sums[i]; }, tiles, target, &before);
    const int v = tile * TILE + (int)threadIdx.x * 4;
    t.load(r, v);
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = t.weight(r, v, 0, j);
    token = token_of(w, v, before, target);
  }
  store_tokens(a, seq, acc, token);
}

int tiles_of(int vocab) { return (vocab + TILE - 1) / TILE; }

}  // namespace

int64_t verify_workspace(int64_t n_seqs, int vocab) {
  const int tiles = tiles_of(vocab);
  return tiles > TILES ? n_seqs * tiles * (int64_t)sizeof(double) : 0;
}

hipError_t launch_verify_drafts(int64_t n_seqs, const VerifyDrafts& a, hipStream_t stream) {
  const int tiles = tiles_of(a.vocab);
  const dim3 seqs((unsigned)n_seqs), block(64 * WAVES);
  if (tiles == 1) {
    hipLaunchKernelGGL(verify_kernel<1>, seqs, block, 0, stream, a);
  } else if (tiles <= TILES) {
    hipLaunchKernelGGL(verify_kernel<TILES>, seqs, block, 0, stream, a);
  } else {
    const int groups = (tiles + TILES - 1) / TILES;
    hipLaunchKernelGGL(verify_sum_kernel, dim3((unsigned)(n_seqs * groups)), block, 0, stream, a, groups, tiles);
    hipLaunchKernelGGL(verify_choose_kernel, seqs, block, 0, stream, a, tiles);
  }
  return hipGetLastError();
}

}  // namespace surge
