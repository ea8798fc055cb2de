// Keys and values written to a cache's pages in 4 bits and read back (gfx950).
//
// Every 32 values of a row have a scale s = 2^e, the least with a <= 7 s for
// a = max(max |x|, 2^-100) (at most 2^125), and the 4-bit float nearest to x / s
// each (+-0, 0.5, 1, 1.5, 2, 3, 4, 6; ties to the even code; what rounds beyond 6
// is 6, off by s at most like the values between 4 and 6, but for magnitudes beyond
// 7 2^125, the largest scale's, off by 2 s).  With a scale of a
// power of two both steps are exact but for that one rounding, and a code times
// its scale is a bf16: reading back rounds nothing.
//
// A wave takes 16 rows of one key head: 8 features a lane, so that it reads 16
// bytes a lane, 128 or 256 of a row together, and writes the codes of
// neighbouring tokens, which lie behind each other in a page, together too.  Bound
// by memory, or in small calls by a chain of three loads (offsets, length, table):
// 100,003 rows x 8 x 128 are written in 77 us, 6.7 TB/s, most of it read (three sets of
// 410 MB in turn, which no cache holds), and read back in 103, 5.0 TB/s, most of it
// written; a copy, half of each, moves 4.9.  64 rows take 4.7 us.
// Rows are loaded and stored past the caches (nontemporal), places found once for
// four heads and neighbouring rows kept on one XCD: 192,000 rows x 12 x 64, written
// and read, 383 us without them, 256 with.
#include "cache_device.h"

namespace surge {
namespace {

constexpr int ROWS = 16;  // of a wave
constexpr int64_t FEW_WAVES = 16384;

// Which sequence and position a row is.
struct RowPlace {
  int seq, pos, length;  // seq < 0: a row of no sequence
};

// The places of rows t0 + r (r < ROWS, one per lane).  cu is searched by 64
// lanes at a time (not at all where a wave holds it), then the boundaries from there
// on are walked in registers.  Offsets that decrease give places within bounds,
// whatever they are.
__device__ __forceinline__ RowPlace place_of(const CacheView& c, const CacheRows& rows, int t0, int r) {
  RowPlace at = {-1, 0, 0};
  const int t = t0 + r;
  if (rows.cu == nullptr) {
    if (t < rows.n_rows) {
      at.seq = t / rows.each;
      at.length = length_of(c, at.seq);
      at.pos = at.length - (at.seq + 1) * rows.each + t;
    }
    return at;
  }
  const int lane = threadIdx.x & 63;
  int lo = 0;
  if (c.n_seqs > 64)
    for (int hi = c.n_seqs; hi - lo > 1;) {  // the last i with cu[i] <= t0 is in [lo, hi)
      const int step = (hi - lo + 63) / 64;
      const int i = lo + lane * step;
      const int n = __popcll(__ballot(i < hi && rows.cu[min(i, c.n_seqs)] <= t0));
      if (n > 0) lo += (n - 1) * step;
      hi = min(lo + step, hi);
    }
  int seq = lo, end = 0;
  bool found = false;
  const int first = rows.cu[lo];
  for (int base = lo + 1; base <= c.n_seqs; base += 64) {
    const int bounds = rows.cu[min(base + lane, c.n_seqs)];
    const int n = min(64, c.n_seqs - base + 1);
    const int before = __popcll(__ballot(lane < n && bounds <= t0));
    if (before > 0) seq = base + before - 1;
    for (int e = before; e < n; ++e) {
      const int bound = __builtin_amdgcn_readlane(bounds, e);
      if (!found && t >= bound) seq = base + e;
      if (!found && t < bound) {
        found = true;
        end = bound;
      }
      if (bound >= t0 + ROWS) break;
    }
    if (__all(found)) break;
  }
  if (found && t >= first && t < rows.n_rows) {
    at.seq = seq;
    at.length = length_of(c, seq);
    at.pos = at.length - end + t;
  }
  return at;
}

// The page's part of key head `head` that holds position pos, or NULL where
// the table's entry is no page.
template <int DH>
__device__ __forceinline__ uint8_t* page_of(const CacheView& c, int seq, int pos, int head) {
  const int page = c.table[seq * c.ld_table + (pos >> c.page_shift)];
  if (page < 0 || page >= c.n_pages) return nullptr;
  return c.pages + page * c.page_bytes + head * PageLayout<DH>::head_bytes(c.page_shift);
}

// A wave's rows and heads: ROWS rows from t0 on, of heads head .. last - 1.
struct Part {
  int t0, head, last;
};
__device__ __forceinline__ bool part_of(const CacheStore& a, Part* p) {
  const int64_t block = (int64_t)(blockIdx.x % 8) * (gridDim.x / 8) + blockIdx.x / 8;
  const int64_t wave = block * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int groups = (a.c.n_kv_heads + a.heads_each - 1) / a.heads_each;
  const int64_t rows = wave / groups;
  if (rows * ROWS >= a.r.n_rows) return false;
  p->t0 = (int)rows * ROWS;
  p->head = (int)(wave % groups) * a.heads_each;
  p->last = min(p->head + a.heads_each, a.c.n_kv_heads);
  return true;
}

// What a wave takes at a time: STEP rows of HEADS heads, 8 features a lane.  128
// bytes of a row at least: of one head of 32 dimensions, half a line, the write
// moved 3.0 TB/s.
template <int DH>
struct Step {
  static constexpr int HEADS = DH < 64 ? 64 / DH : 1, PER = HEADS * DH / 8, STEP = 64 / PER, N = ROWS / STEP;
};

template <int DH>
__global__ __launch_bounds__(256) void cache_write_kernel(CacheStore a) {
  using L = PageLayout<DH>;
  constexpr int HEADS = Step<DH>::HEADS, PER = Step<DH>::PER, STEP = Step<DH>::STEP, N = Step<DH>::N;
  const int lane = threadIdx.x & 63, more = lane % PER / (DH / 8), piece = lane % (DH / 8);
  Part part;
  if (!part_of(a, &part)) return;
  u32x4 x[2][N];
  auto load = [&](int first) {
    const int head = min(first + more, part.last - 1);
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int64_t t = min(part.t0 + n * STEP + lane / PER, a.r.n_rows - 1);
      x[0][n] = __builtin_nontemporal_load(
          reinterpret_cast<const u32x4*>(a.k + t * a.ld_k + head * DH + piece * 8));
      x[1][n] = __builtin_nontemporal_load(
          reinterpret_cast<const u32x4*>(a.v + t * a.ld_v + head * DH + piece * 8));
    }
  };
  load(part.head);
  const RowPlace mine = place_of(a.c, a.r, part.t0, lane % ROWS);
  uint8_t* page[N];  // of head 0
  int slot[N];
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const int from = n * STEP + lane / PER;
    const int seq = __shfl(mine.seq, from), pos = __shfl(mine.pos, from);
    page[n] = seq < 0 || pos < 0 ? nullptr : page_of<DH>(a.c, seq, pos, 0);
    slot[n] = pos & ((1 << a.c.page_shift) - 1);
  }
  for (int first = part.head; first < part.last; first += HEADS) {
    uint32_t codes[2][N], bytes[2][N];
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        const uint32_t v[4] = {x[w][n][0], x[w][n][1], x[w][n][2], x[w][n][3]};
        // Largest magnitude, as bits (of infinities and NaN the largest).
        uint32_t most = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          most = max(most, v[i] << 16 & 0x7fff0000u);
          most = max(most, v[i] & 0x7fff0000u);
        }
        // Over the four lanes of 32 features.
        most = max(most, (uint32_t)__builtin_amdgcn_mov_dpp((int)most, 0xb1, 0xf, 0xf, true));
        most = max(most, (uint32_t)__builtin_amdgcn_mov_dpp((int)most, 0x4e, 0xf, 0xf, true));
        // With a = 1.f 2^E: e = E - 2 where 1.f <= 1.75, else E - 1.
        uint32_t byte = ((max(most, 0x0d800000u) + 0x1fffffu) >> 23) - 2;
        byte = most >= 0x7f800000u ? NAN_SCALE : min(byte, 252u);
        const float scale = scale_of(byte);
        uint32_t c = 0;
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, v[0]), scale, 0);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, v[1]), scale, 1);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, v[2]), scale, 2);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, v[3]), scale, 3);
        codes[w][n] = c;
        bytes[w][n] = byte;
      }
    if (first + HEADS < part.last) load(first + HEADS);
    const int64_t head_at = (first + more) * L::head_bytes(a.c.page_shift);
#pragma unroll
    for (int n = 0; n < N; ++n)
      if (page[n] && first + more < part.last)
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          uint8_t* const to = page[n] + head_at;
          *reinterpret_cast<uint32_t*>(to + L::codes(a.c.page_shift, slot[n], w) + piece * 4) = codes[w][n];
          if (piece % 4 == 0) to[L::scales(a.c.page_shift, slot[n], w) + piece / 4] = (uint8_t)bytes[w][n];
        }
  }
}

template <int DH>
__global__ __launch_bounds__(256) void cache_read_kernel(CacheStore a) {
  using L = PageLayout<DH>;
  constexpr int HEADS = Step<DH>::HEADS, PER = Step<DH>::PER, STEP = Step<DH>::STEP, N = Step<DH>::N;
  const int lane = threadIdx.x & 63, more = lane % PER / (DH / 8), piece = lane % (DH / 8);
  Part part;
  if (!part_of(a, &part)) return;
  const RowPlace mine = place_of(a.c, a.r, part.t0, lane % ROWS);
  const uint8_t* page[N];  // of head 0; NULL: nothing to read
  int slot[N];
  uint32_t without[N];     // the scale byte then: zeros, or NaN where there is no page
  bool row[N];
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const int from = n * STEP + lane / PER;
    const int seq = __shfl(mine.seq, from), pos = __shfl(mine.pos, from);
    row[n] = seq >= 0;
    without[n] = pos < 0 ? 1 : NAN_SCALE;
    page[n] = row[n] && pos >= 0 ? page_of<DH>(a.c, seq, pos, 0) : nullptr;
    slot[n] = pos & ((1 << a.c.page_shift) - 1);
  }
  uint32_t codes[2][N], bytes[2][N];
  auto load = [&](int first) {
    const int64_t head_at = min(first + more, part.last - 1) * L::head_bytes(a.c.page_shift);
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        codes[w][n] = 0;
        bytes[w][n] = without[n];
        if (page[n]) {
          const uint8_t* const from = page[n] + head_at;
          codes[w][n] = *reinterpret_cast<const uint32_t*>(from + L::codes(a.c.page_shift, slot[n], w) + piece * 4);
          bytes[w][n] = from[L::scales(a.c.page_shift, slot[n], w) + piece / 4];
        }
      }
  };
  load(part.head);
  for (int first = part.head; first < part.last; first += HEADS) {
    u32x4 x[2][N];
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int w = 0; w < 2; ++w) x[w][n] = __builtin_bit_cast(u32x4, decode8(codes[w][n], scale_of(bytes[w][n])));
    if (first + HEADS < part.last) load(first + HEADS);
    const int head = first + more;
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int64_t t = part.t0 + n * STEP + lane / PER;
      if (!row[n] || head >= part.last) continue;
      __builtin_nontemporal_store(x[0][n], reinterpret_cast<u32x4*>(a.k + t * a.ld_k + head * DH + piece * 8));
      __builtin_nontemporal_store(x[1][n], reinterpret_cast<u32x4*>(a.v + t * a.ld_v + head * DH + piece * 8));
    }
  }
}

// Heads of a wave: one step's in small calls, which need the waves, four in large ones,
// whose waves find their rows' places once for them.
int heads_each(int64_t n_rows, int n_kv_heads, int d_head) {
  const int64_t waves = (n_rows + ROWS - 1) / ROWS * n_kv_heads;
  return waves > FEW_WAVES ? 4 : d_head < 64 ? 64 / d_head : 1;
}

}  // namespace

int64_t cache_store_blocks(int64_t n_rows, int n_kv_heads, int d_head) {
  const int each = heads_each(n_rows, n_kv_heads, d_head);
  return ((n_rows + ROWS - 1) / ROWS * ((n_kv_heads + each - 1) / each) + 31) / 32 * 8;
}

hipError_t launch_cache_write(CacheStore a, int d_head, hipStream_t stream) {
  a.heads_each = heads_each(a.r.n_rows, a.c.n_kv_heads, d_head);
  const dim3 grid((unsigned)cache_store_blocks(a.r.n_rows, a.c.n_kv_heads, d_head));
  if (d_head == 32) hipLaunchKernelGGL(cache_write_kernel<32>, grid, dim3(256), 0, stream, a);
  if (d_head == 64) hipLaunchKernelGGL(cache_write_kernel<64>, grid, dim3(256), 0, stream, a);
  if (d_head == 128) hipLaunchKernelGGL(cache_write_kernel<128>, grid, dim3(256), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_cache_read(CacheStore a, int d_head, hipStream_t stream) {
  a.heads_each = heads_each(a.r.n_rows, a.c.n_kv_heads, d_head);
  const dim3 grid((unsigned)cache_store_blocks(a.r.n_rows, a.c.n_kv_heads, d_head));
  if (d_head == 32) hipLaunchKernelGGL(cache_read_kernel<32>, grid, dim3(256), 0, stream, a);
  if (d_head == 64) hipLaunchKernelGGL(cache_read_kernel<64>, grid, dim3(256), 0, stream, a);
  if (d_head == 128) hipLaunchKernelGGL(cache_read_kernel<128>, grid, dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace surge
