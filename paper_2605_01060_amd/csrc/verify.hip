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
//
// A small call is a chain of latencies: the drafts, their probabilities, the row,
// then sums and scans.  Those are lane exchanges in registers and two barriers,
// each wave finding the tile and the wave that the sum passes in for itself (through
// LDS 15.7 us a call, so 7.5, most of it the caller's).  256 x 6 drafts of 100,003
// tokens take 43 us, 37 of them the sums, 5.5 TB/s; with a workgroup a sequence, row
// by row, 133.
#include "cache_device.h"

namespace surge {
namespace {

constexpr int WAVES = 16, TILE = 64 * WAVES * 4, TILES = 8;

// A double's value in another lane by a DPP control; lanes that the control or
// the row mask leaves out get 0.
template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ double dpp64(double v) {
  const uint64_t bits = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)bits, CTRL, ROWS, 0xf, true);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(bits >> 32), CTRL, ROWS, 0xf, true);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
constexpr int XOR1 = 0xb1, XOR2 = 0x4e, HALF_MIRROR = 0x141, SHR = 0x110, ROR8 = 0x128, BCAST15 = 0x142,
              BCAST31 = 0x143;

// a and b are exchanged between lanes 32 (16) apart and added: the lower lanes
// (rows 0 and 2) get the sum of a's two, the others of b's.
__device__ __forceinline__ double swap_add32(double a, double b) {
  const uint64_t x = __builtin_bit_cast(uint64_t, a), y = __builtin_bit_cast(uint64_t, b);
  const auto lo = __builtin_amdgcn_permlane32_swap((uint32_t)x, (uint32_t)y, false, false);
  const auto hi = __builtin_amdgcn_permlane32_swap((uint32_t)(x >> 32), (uint32_t)(y >> 32), false, false);
  return __builtin_bit_cast(double, (uint64_t)hi[0] << 32 | lo[0]) +
         __builtin_bit_cast(double, (uint64_t)hi[1] << 32 | lo[1]);
}
__device__ __forceinline__ double swap_add16(double a, double b) {
  const uint64_t x = __builtin_bit_cast(uint64_t, a), y = __builtin_bit_cast(uint64_t, b);
  const auto lo = __builtin_amdgcn_permlane16_swap((uint32_t)x, (uint32_t)y, false, false);
  const auto hi = __builtin_amdgcn_permlane16_swap((uint32_t)(x >> 32), (uint32_t)(y >> 32), false, false);
  return __builtin_bit_cast(double, (uint64_t)hi[0] << 32 | lo[0]) +
         __builtin_bit_cast(double, (uint64_t)hi[1] << 32 | lo[1]);
}

// The wave's sums of N values, written to to[0 .. N-1].
template <int N>
__device__ __forceinline__ void wave_sums_to(const double* s, double* to) {
  static_assert(N == 1 || N == 8, "one value, or eight that share the exchanges");
  const int lane = threadIdx.x & 63;
  double v;
  int which = 0;
  if constexpr (N == 8) {
    double a[4], b[2];
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] = swap_add32(s[2 * i], s[2 * i + 1]);
#pragma unroll
    for (int i = 0; i < 2; ++i) b[i] = swap_add16(a[2 * i], a[2 * i + 1]);
    const bool second = lane & 8;
    v = (second ? b[1] : b[0]) + dpp64<ROR8>(second ? b[0] : b[1]);
    which = (lane >> 5) + (lane >> 4 & 1) * 2 + (lane >> 3 & 1) * 4;
  } else {
    v = swap_add32(s[0], s[0]);
    v = swap_add16(v, v);
    v += dpp64<ROR8>(v);
  }
  v += dpp64<HALF_MIRROR>(v);
  v += dpp64<XOR1>(v);
  v += dpp64<XOR2>(v);
  if ((lane & 7) == 0 && (N == 8 || lane == 0)) to[which] = v;
}

// Sum of a lane and those before it in its row of 16, in the wave.
__device__ __forceinline__ double scan16(double v) {
  v += dpp64<SHR + 1>(v);
  v += dpp64<SHR + 2>(v);
  v += dpp64<SHR + 4>(v);
  return v + dpp64<SHR + 8>(v);
}
__device__ __forceinline__ double scan64(double v) {
  v = scan16(v);
  v += dpp64<BCAST15, 0xa>(v);
  return v + dpp64<BCAST31, 0xc>(v);
}

__device__ __forceinline__ double lane_of(double v, int lane) {
  const uint64_t bits = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)bits, lane);
  const uint32_t hi = __builtin_amdgcn_readlane((int)(uint32_t)(bits >> 32), lane);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}

// The drafts of a sequence that are accepted, looked at by a wave: the first
// that is not ends them.  *n: how many there are.
__device__ __forceinline__ int accepted_drafts(const VerifyDrafts& a, int64_t seq, int* n) {
  const int lane = threadIdx.x & 63;
  const int given = a.n_drafts ? a.n_drafts[seq] : a.max_drafts;
  int acc = -1;
  for (int j0 = 0; j0 < a.max_drafts && acc < 0; j0 += 64) {
    const int j = j0 + lane;
    bool ok = false;
    if (j < a.max_drafts) {
      const int x = a.drafts[seq * a.max_drafts + j];
      const double u = a.u[seq * (a.max_drafts + 1) + j];
      if (x >= 0 && x < a.vocab) {
        const double p = a.p[(seq * (a.max_drafts + 1) + j) * a.ld_p + x];
        const double q = a.q ? (double)a.q[(seq * a.max_drafts + j) * a.ld_q + x] : 1.0;
        ok = u * q < p;
      }
    }
    const uint64_t failed = ~__ballot(ok && j < given);
    if (failed) acc = j0 + __builtin_ctzll(failed);
  }
  *n = __builtin_amdgcn_readfirstlane(min(max(given, 0), a.max_drafts));
  return __builtin_amdgcn_readfirstlane(acc < 0 ? *n : min(acc, *n));
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

__device__ __forceinline__ Row row_of(const VerifyDrafts& a, int64_t seq, int acc, bool rejected) {
  Row r;
  r.has_q = rejected && a.q;
  r.p = row_buffer(a.p + (seq * (a.max_drafts + 1) + acc) * a.ld_p, a.vocab);
  r.q = row_buffer(r.has_q ? a.q + (seq * a.max_drafts + acc) * a.ld_q : nullptr, a.vocab);
  r.without = rejected && !a.q ? a.drafts[seq * a.max_drafts + acc] : -1;
  return r;
}

__device__ __forceinline__ f32x4 load4(__amdgpu_buffer_rsrc_t row, int v) {
  return __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(row, v * 4, 0, 0));
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

// Of values in lanes (a lane's own and the sum up to it), the first lane with a
// value at which the sum passes the target, else the last with a value.
__device__ __forceinline__ int passing_lane(double value, double upto, double target) {
  const uint64_t some = __ballot(value > 0.0), over = __ballot(value > 0.0 && upto > target);
  return over ? __builtin_ctzll(over) : some ? 63 - __builtin_clzll(some) : 0;
}

__device__ __forceinline__ bool drawable(double total) { return total > 0.0 && total < HUGE_VAL; }

__device__ __forceinline__ double target_of(const VerifyDrafts& a, int64_t seq, double total) {
  return (double)a.u[seq * (a.max_drafts + 1) + a.max_drafts] * total;
}

// The accepted drafts, the token, -1, by one wave.
__device__ __forceinline__ void store_tokens(const VerifyDrafts& a, int64_t seq, int acc, int token) {
  const int lane = threadIdx.x & 63;
  for (int j = lane; j <= a.max_drafts; j += 64)
    a.tokens[seq * (a.max_drafts + 1) + j] = j < acc ? a.drafts[seq * a.max_drafts + j] : j == acc ? token : -1;
  if (lane == 0) a.accepted[seq] = acc;
}

// Finds and stores the token of a tile, of which this thread's four from v on
// weigh w and the tiles before it `before`: the wave in which the sum passes the
// target does.
__device__ __forceinline__ void choose_token(const VerifyDrafts& a, int64_t seq, int acc, const double* w, int v,
                                             double before, double target) {
  __shared__ double shared[WAVES];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const double s = (w[0] + w[1]) + (w[2] + w[3]);
  const double upto = scan64(s);
  if (lane == 63) shared[wave] = upto;
  __syncthreads();
  const double of_wave = lane < WAVES ? shared[lane] : 0.0;
  const double waves = before + scan16(of_wave);
  const int its = passing_lane(of_wave, waves, target);
  if (its != wave) return;
  const double start = its > 0 ? lane_of(waves, its - 1) : before;
  const int at = passing_lane(s, start + upto, target);
  double c = start + (upto - s);
  int token = -1;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if (w[j] > 0.0 && (token < 0 || !(c > target))) token = v + j;
    c += w[j];
  }
  store_tokens(a, seq, acc, __builtin_amdgcn_readlane(token, at));
}

// A vocabulary of at most N tiles: a workgroup a sequence, its row in registers.
template <int N>
__global__ __launch_bounds__(64 * WAVES) void verify_kernel(VerifyDrafts a) {
  __shared__ double shared[WAVES][N];
  const int64_t seq = blockIdx.x;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, v = (int)threadIdx.x * 4;
  int n;
  const int acc = accepted_drafts(a, seq, &n);
  Row r = row_of(a, seq, acc, acc < n);
  Tokens<N> t;
  t.load(r, v);
  double of_tile, upto, total;
  while (true) {
    double s[N];
#pragma unroll
    for (int i = 0; i < N; ++i) s[i] = t.sum(r, v, i);
    wave_sums_to<N>(s, shared[wave]);
    __syncthreads();
    // Lane l sums tile l % 8 (or the only one) over all waves.
    double x = 0.0;
    if constexpr (N == 8) {
      x = shared[lane >> 3][lane & 7] + shared[8 + (lane >> 3)][lane & 7];
      x += dpp64<ROR8>(x);
    } else {
      x = shared[lane & 15][0];
      x += dpp64<ROR8>(x);
      x += dpp64<HALF_MIRROR>(x);
      x += dpp64<XOR1>(x);
      x += dpp64<XOR2>(x);
      x *= 0.25;  // the four rows of lanes have the same
    }
    x = swap_add16(x, x);
    x = swap_add32(x, x);
    of_tile = lane < N ? x : 0.0;
    upto = scan16(of_tile);
    total = lane_of(upto, N - 1);
    if (total > 0.0 || (!r.has_q && r.without < 0)) break;
    // Nothing left over by q: the target's own probabilities.
    r.has_q = false;
    r.without = -1;
#pragma unroll
    for (int i = 0; i < N; ++i) t.q[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    __syncthreads();  // the sums are read before they are made again
  }
  if (!drawable(total)) {
    if (wave == 0) store_tokens(a, seq, acc, -1);
    return;
  }
  const double target = target_of(a, seq, total);
  const int tile = passing_lane(of_tile, upto, target);
  const double before = tile > 0 ? lane_of(upto, tile - 1) : 0.0;
  Tokens<1> one = {{t.p[0]}, {t.q[0]}};
#pragma unroll
  for (int i = 1; i < N; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      one.p[0][j] = i == tile ? t.p[i][j] : one.p[0][j];
      one.q[0][j] = i == tile ? t.q[i][j] : one.q[0][j];
    }
  double w[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) w[j] = one.weight(r, v + tile * TILE, 0, j);
  choose_token(a, seq, acc, w, v + tile * TILE, before, target);
}

// The tiles' sums of the row that decides, a workgroup for each TILES of them, and
// 2 accepted drafts + (one is rejected) of a sequence.
__global__ __launch_bounds__(64 * WAVES) void verify_sum_kernel(VerifyDrafts a, int groups, int tiles, int* taken) {
  __shared__ double shared[WAVES][TILES];
  const int64_t seq = blockIdx.x / (unsigned)groups;
  const int first = (int)(blockIdx.x % (unsigned)groups) * TILES;
  const int v = first * TILE + (int)threadIdx.x * 4;
  int n;
  const int acc = accepted_drafts(a, seq, &n);
  const Row r = row_of(a, seq, acc, acc < n);
  if (first == 0 && threadIdx.x == 0) taken[seq] = 2 * acc + (acc < n);
  Tokens<TILES> t;
  t.load(r, v);
  double s[TILES];
#pragma unroll
  for (int i = 0; i < TILES; ++i) s[i] = t.sum(r, v, i);
  wave_sums_to<TILES>(s, shared[threadIdx.x >> 6]);
  __syncthreads();
  if (threadIdx.x < TILES && first + (int)threadIdx.x < tiles) {
    double x = 0.0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) x += shared[w][threadIdx.x];
    a.sums[seq * tiles + first + threadIdx.x] = x;
  }
}

__global__ __launch_bounds__(64 * WAVES) void verify_choose_kernel(VerifyDrafts a, int tiles, const int* taken) {
  __shared__ double shared[WAVES][1];
  const int64_t seq = blockIdx.x;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  double* const sums = a.sums + seq * tiles;
  const int mark = taken[seq], acc = mark >> 1;
  Row r = row_of(a, seq, acc, mark & 1);
  double total = 0.0;
  for (int i = 0; i < tiles; i += 64) total += lane_of(scan64(i + lane < tiles ? sums[i + lane] : 0.0), 63);
  Tokens<1> t;
  if (!(total > 0.0) && (r.has_q || r.without >= 0)) {
    // Nothing left over by q: the target's own probabilities.
    r.q = row_buffer(nullptr, 0);
    r.without = -1;
    total = 0.0;
    for (int i = 0; i < tiles; ++i) {
      const int v = i * TILE + (int)threadIdx.x * 4;
      t.load(r, v);
      const double s = t.sum(r, v, 0);
      __syncthreads();  // the last tile's sums are read
      wave_sums_to<1>(&s, shared[wave]);
      __syncthreads();
      double x = 0.0;
      for (int w = 0; w < WAVES; ++w) x += shared[w][0];
      if (threadIdx.x == 0) sums[i] = x;
      total += x;
    }
    __syncthreads();
  }
  if (!drawable(total)) {
    if (wave == 0) store_tokens(a, seq, acc, -1);
    return;
  }
  const double target = target_of(a, seq, total);
  int tile = 0;
  double upto_here = 0.0, before = 0.0;
  for (int i = 0; i < tiles; i += 64) {
    const double x = i + lane < tiles ? sums[i + lane] : 0.0;
    const double upto = upto_here + scan64(x);
    if (__any(x > 0.0)) {
      const int at = passing_lane(x, upto, target);
      tile = i + at;
      before = at > 0 ? lane_of(upto, at - 1) : upto_here;
      if (lane_of(upto, at) > target) break;
    }
    upto_here = lane_of(upto, 63);
  }
  const int v = tile * TILE + (int)threadIdx.x * 4;
  t.load(r, v);
  double w[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) w[j] = t.weight(r, v, 0, j);
  choose_token(a, seq, acc, w, v, before, target);
}

int tiles_of(int vocab) { return (vocab + TILE - 1) / TILE; }

}  // namespace

int64_t verify_workspace(int64_t n_seqs, int vocab) {
  const int tiles = tiles_of(vocab);
  return tiles > TILES ? n_seqs * (tiles * (int64_t)sizeof(double) + (int64_t)sizeof(int)) : 0;
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
    int* const taken = reinterpret_cast<int*>(a.sums + n_seqs * tiles);
    hipLaunchKernelGGL(verify_sum_kernel, dim3((unsigned)(n_seqs * groups)), block, 0, stream, a, groups, tiles, taken);
    hipLaunchKernelGGL(verify_choose_kernel, seqs, block, 0, stream, a, tiles, taken);
  }
  return hipGetLastError();
}

}  // namespace surge
