// Entry points of a decoder's operators: argument checks and launches of the
// cache's write and read, of attention over it and of the check of drafts.
#include <math.h>

#include <algorithm>

#include "cache.h"
#include "checks.h"
#include "surge_ops.h"

using namespace surge;

namespace {

// Positions are counted in 32 bits, a block of keys beyond the last one too.
constexpr int64_t kMostLength = 1 << 30;
constexpr int kMaxSeqs = 1 << 20, kMaxHeads = 1024, kMaxDrafts = 1024;
constexpr int kMaxVocab = 1 << 22;
// Threads of a launch are a 32-bit number.
constexpr int64_t kMostThreads = 1ll << 31;

int64_t head_bytes(const surge_kv_cache* c) {
  return (int64_t)c->page_tokens * c->d_head / 16 * 17;
}

surge_status check_geometry(int32_t page_tokens, int32_t n_kv_heads, int32_t d_head) {
  if (page_tokens < 16 || page_tokens > 256 || (page_tokens & (page_tokens - 1)))
    return fail(SURGE_ERR_INVALID_ARGUMENT, "page_tokens=%d: 16, 32, 64, 128 or 256 are needed",
                page_tokens);
  if (n_kv_heads < 1 || n_kv_heads > kMaxHeads)
    return fail(SURGE_ERR_INVALID_ARGUMENT, "n_kv_heads=%d outside [1, %d]", n_kv_heads, kMaxHeads);
  if (d_head != 32 && d_head != 64 && d_head != 128)
    return fail(SURGE_ERR_INVALID_ARGUMENT, "d_head=%d", d_head);
  return SURGE_OK;
}

// What does not depend on the device's memory.
surge_status check_cache(const surge_kv_cache* c) {
  if (!c) return fail(SURGE_ERR_INVALID_ARGUMENT, "cache is NULL");
  CHECK(check_geometry(c->page_tokens, c->n_kv_heads, c->d_head));
  if (c->n_seqs < 0 || c->n_seqs > kMaxSeqs)
    return fail(SURGE_ERR_INVALID_ARGUMENT, "n_seqs=%d outside [0, %d]", c->n_seqs, kMaxSeqs);
  if (c->n_pages < 1 || c->n_pages > (int64_t)INT32_MAX)
    return fail(SURGE_ERR_INVALID_ARGUMENT, "n_pages=%lld outside [1, 2^31)", (long long)c->n_pages);
  if (c->max_length < 0 || c->max_length > kMostLength)
    return fail(SURGE_ERR_INVALID_ARGUMENT, "max_length=%lld outside [0, 2^30]", (long long)c->max_length);
  const int64_t entries = (c->max_length + c->page_tokens - 1) / c->page_tokens;
  if (c->ld_table < entries || c->ld_table > kMostLength)
    return fail(SURGE_ERR_INVALID_ARGUMENT, "rows of %lld table entries: max_length needs %lld",
                (long long)c->ld_table, (long long)entries);
  return SURGE_OK;
}

surge_status check_memory(const surge_kv_cache* c) {
  CHECK(check_vector("pages", c->d_pages, true));
  if (!c->d_table || !c->d_lengths || !aligned(c->d_table, 4) || !aligned(c->d_lengths, 4))
    return fail(SURGE_ERR_INVALID_ARGUMENT, "table and lengths are needed, 4-byte aligned");
  return SURGE_OK;
}

// Rows of a call over the cache's sequences.
surge_status check_call_rows(const surge_kv_cache* c, int64_t n_rows, const int32_t* d_cu) {
  if (n_rows < 0 || n_rows > kMostLength)
    return fail(SURGE_ERR_INVALID_ARGUMENT, "n_rows=%lld outside [0, 2^30]", (long long)n_rows);
  if (!aligned(d_cu, 4)) return fail(SURGE_ERR_INVALID_ARGUMENT, "cu must be 4-byte aligned");
  if (!d_cu && c->n_seqs > 0 && n_rows % c->n_seqs)
    return fail(SURGE_ERR_INVALID_ARGUMENT, "%lld rows without cu: a multiple of n_seqs=%d is needed",
                (long long)n_rows, c->n_seqs);
  return SURGE_OK;
}

CacheView view_of(const surge_kv_cache* c) {
  CacheView v;
  v.pages = c->d_pages;
  v.n_pages = c->n_pages;
  v.page_bytes = head_bytes(c) * c->n_kv_heads;
  v.page_shift = __builtin_ctz(c->page_tokens);
  v.n_kv_heads = c->n_kv_heads;
  v.n_seqs = c->n_seqs;
  v.max_length = (int)c->max_length;
  v.table = c->d_table;
  v.ld_table = c->ld_table;
  v.lengths = c->d_lengths;
  return v;
}

CacheRows rows_of(const surge_kv_cache* c, int64_t n_rows, const int32_t* d_cu) {
  return {d_cu, (int)n_rows, (int)(n_rows / c->n_seqs)};
}

surge_status store(bool write, const surge_kv_cache* cache, int64_t n_rows, const int32_t* d_cu,
                   const uint16_t* d_k, int64_t ld_k, const uint16_t* d_v, int64_t ld_v, void* hip_stream) {
  clear_error();
  CHECK(check_cache(cache));
  CHECK(check_call_rows(cache, n_rows, d_cu));
  if (n_rows == 0 || cache->n_seqs == 0) return SURGE_OK;
  CHECK(check_memory(cache));
  const int64_t cols = (int64_t)cache->n_kv_heads * cache->d_head;
  CHECK(check_matrix("k", d_k, cols, ld_k, 8));
  CHECK(check_matrix("v", d_v, cols, ld_v, 8));
  if (d_k == d_v && !write) return fail(SURGE_ERR_INVALID_ARGUMENT, "k is v");
  if ((const void*)d_k == cache->d_pages || (const void*)d_v == cache->d_pages)
    return fail(SURGE_ERR_INVALID_ARGUMENT, "k or v is pages");
  if (cache_store_blocks(n_rows, cache->n_kv_heads, cache->d_head) > kMostThreads / 256)
    return fail(SURGE_ERR_CAPACITY, "too many rows and heads for one call");
  int dev = 0, n_cus = 0;
  CHECK(current_device((hipStream_t)hip_stream, &dev, &n_cus));
  const CacheStore a = {view_of(cache), rows_of(cache, n_rows, d_cu), const_cast<uint16_t*>(d_k),
                        const_cast<uint16_t*>(d_v), ld_k, ld_v, 1};
  HIP_TRY(write ? launch_cache_write(a, cache->d_head, (hipStream_t)hip_stream)
                : launch_cache_read(a, cache->d_head, (hipStream_t)hip_stream));
  return SURGE_OK;
}

// The cut of a call and the workspace that it needs.
surge_status attention_shape(const surge_kv_cache* c, int64_t max_rows, int32_t n_heads, int n_cus,
                             CacheShape* s, int64_t* bytes) {
  *s = cache_attention_shape(c->n_seqs, max_rows, c->n_kv_heads, n_heads / c->n_kv_heads, c->d_head,
                             c->max_length, n_cus);
  // (Units that are shared out, and with them the rows of their join, are few.)
  if ((s->wave_units ? (s->units + 3) / 4 : s->units) > kMostThreads / 256)
    return fail(SURGE_ERR_CAPACITY, "too many rows, heads and sequences for one call");
  *bytes = s->workspace_bytes(c->d_head);
  return SURGE_OK;
}

surge_status check_heads(const surge_kv_cache* c, int64_t max_rows, int32_t n_heads) {
  if (n_heads < 1 || n_heads > kMaxHeads || n_heads % c->n_kv_heads)
    return fail(SURGE_ERR_INVALID_ARGUMENT, "n_heads=%d, n_kv_heads=%d", n_heads, c->n_kv_heads);
  if (max_rows < 0 || max_rows > kMostLength / n_heads)
    return fail(SURGE_ERR_INVALID_ARGUMENT, "max_rows=%lld", (long long)max_rows);
  return SURGE_OK;
}

}  // namespace

extern "C" {

surge_status surge_cache_page_bytes(int32_t page_tokens, int32_t n_kv_heads, int32_t d_head,
                                    int64_t* bytes) {
  clear_error();
  if (!bytes) return fail(SURGE_ERR_INVALID_ARGUMENT, "bytes is NULL");
  CHECK(check_geometry(page_tokens, n_kv_heads, d_head));
  *bytes = (int64_t)page_tokens * d_head / 16 * 17 * n_kv_heads;
  return SURGE_OK;
}

surge_status surge_op_cache_write(const surge_kv_cache* cache, int64_t n_rows, const int32_t* d_cu,
                                  const uint16_t* d_k, int64_t ld_k, const uint16_t* d_v, int64_t ld_v,
                                  void* hip_stream) {
  return store(true, cache, n_rows, d_cu, d_k, ld_k, d_v, ld_v, hip_stream);
}

surge_status surge_op_cache_read(const surge_kv_cache* cache, int64_t n_rows, const int32_t* d_cu,
                                 uint16_t* d_k, int64_t ld_k, uint16_t* d_v, int64_t ld_v,
                                 void* hip_stream) {
  return store(false, cache, n_rows, d_cu, d_k, ld_k, d_v, ld_v, hip_stream);
}

surge_status surge_cache_attention_workspace(const surge_kv_cache* cache, int64_t max_rows,
                                             int32_t n_heads, int64_t* bytes) {
  clear_error();
  if (!bytes) return fail(SURGE_ERR_INVALID_ARGUMENT, "bytes is NULL");
  *bytes = 0;
  CHECK(check_cache(cache));
  CHECK(check_heads(cache, max_rows, n_heads));
  if (max_rows == 0 || cache->n_seqs == 0) return SURGE_OK;
  int dev = 0, n_cus = 0;
  CHECK(current_device(nullptr, &dev, &n_cus));
  CacheShape s;
  return attention_shape(cache, max_rows, n_heads, n_cus, &s, bytes);
}

surge_status surge_op_cache_attention(const surge_kv_cache* cache, int64_t n_rows, const int32_t* d_cu,
                                      int64_t max_rows, int32_t n_heads, int32_t causal, float scale,
                                      const uint16_t* d_q, int64_t ld_q, void* d_workspace,
                                      int64_t workspace_bytes, uint16_t* d_out, int64_t ld_out,
                                      void* hip_stream) {
  clear_error();
  CHECK(check_cache(cache));
  CHECK(check_call_rows(cache, n_rows, d_cu));
  CHECK(check_heads(cache, max_rows, n_heads));
  if (causal != 0 && causal != 1) return fail(SURGE_ERR_INVALID_ARGUMENT, "causal=%d", causal);
  // Times log2(e) it is still a float.
  const float scale_log2 = scale * 1.4426950408889634f;
  if (!(scale > 0.0f) || !isfinite(scale_log2))
    return fail(SURGE_ERR_INVALID_ARGUMENT, "scale=%g must be positive and below 2^127", (double)scale);
  if (n_rows == 0 || cache->n_seqs == 0) return SURGE_OK;
  if (max_rows < 1 || (!d_cu && n_rows > max_rows * cache->n_seqs))
    return fail(SURGE_ERR_INVALID_ARGUMENT, "max_rows=%lld is less than a sequence's rows",
                (long long)max_rows);
  CHECK(check_memory(cache));
  const int64_t cols = (int64_t)n_heads * cache->d_head;
  CHECK(check_matrix("q", d_q, cols, ld_q, 8));
  CHECK(check_matrix("out", d_out, cols, ld_out, 8));
  CHECK(check_place("out", d_out, 0, "q", d_q, 0, false));
  CHECK(check_place("out", d_out, 0, "pages", cache->d_pages, 0, false));
  int dev = 0, n_cus = 0;
  CHECK(current_device((hipStream_t)hip_stream, &dev, &n_cus));
  CacheShape s;
  int64_t need = 0;
  CHECK(attention_shape(cache, max_rows, n_heads, n_cus, &s, &need));
  if (need > 0) {
    CHECK(check_vector("workspace", d_workspace, true));
    if (workspace_bytes < need)
      return fail(SURGE_ERR_CAPACITY, "workspace of %lld bytes, %lld are needed",
                  (long long)workspace_bytes, (long long)need);
  }
  CacheAttention a;
  a.c = view_of(cache);
  a.r = rows_of(cache, n_rows, d_cu);
  a.q = d_q;
  a.out = d_out;
  a.ld_q = ld_q;
  a.ld_out = ld_out;
  a.group = n_heads / cache->n_kv_heads;
  a.max_rows = (int)max_rows;
  a.causal = causal != 0;
  a.scale_log2 = scale_log2;
  a.tile_rows = s.tile_rows;
  a.block_shift = s.block_shift;
  a.tiles = (int)s.tiles;
  a.units = (int)s.units;
  a.workers = (int)s.workers;
  a.by_group = divisor(a.group);
  a.by_tiles = divisor(a.tiles);
  a.by_heads = divisor(cache->n_kv_heads);
  a.by_units = divisor(cache->n_seqs * cache->n_kv_heads);
  a.by_workers = divisor(std::max(a.workers, 1));
  a.least_share = s.least_share;
  a.join_waves = s.workers ? cache_attention_join(s, cache->max_length) : 0;
  a.wave_units = s.wave_units;
  a.part_o = (float*)d_workspace;
  a.part_ml = (float2*)(a.part_o + s.slot_rows() * cache->d_head);
  a.joins = (int2*)(a.part_ml + s.slot_rows());
  HIP_TRY(launch_cache_attention(a, cache->d_head, (hipStream_t)hip_stream));
  return SURGE_OK;
}

surge_status surge_verify_workspace(int64_t n_seqs, int32_t vocab, int64_t* bytes) {
  clear_error();
  if (!bytes) return fail(SURGE_ERR_INVALID_ARGUMENT, "bytes is NULL");
  *bytes = 0;
  if (n_seqs < 0 || n_seqs > kMaxSeqs || vocab < 1 || vocab > kMaxVocab)
    return fail(SURGE_ERR_INVALID_ARGUMENT, "n_seqs=%lld, vocab=%d", (long long)n_seqs, vocab);
  *bytes = verify_workspace(n_seqs, vocab);
  return SURGE_OK;
}

surge_status surge_op_verify_drafts(int64_t n_seqs, int32_t max_drafts, int32_t vocab,
                                    const int32_t* d_n_drafts, const int32_t* d_drafts, const float* d_p,
                                    int64_t ld_p, const float* d_q, int64_t ld_q, const float* d_u,
                                    void* d_workspace, int64_t workspace_bytes, int32_t* d_tokens,
                                    int32_t* d_accepted, void* hip_stream) {
  clear_error();
  if (n_seqs < 0 || n_seqs > kMaxSeqs)
    return fail(SURGE_ERR_INVALID_ARGUMENT, "n_seqs=%lld outside [0, 2^20]", (long long)n_seqs);
  if (max_drafts < 0 || max_drafts > kMaxDrafts)
    return fail(SURGE_ERR_INVALID_ARGUMENT, "max_drafts=%d outside [0, %d]", max_drafts, kMaxDrafts);
  if (vocab < 1 || vocab > kMaxVocab)
    return fail(SURGE_ERR_INVALID_ARGUMENT, "vocab=%d outside [1, 2^22]", vocab);
  if (n_seqs == 0) return SURGE_OK;
  const struct {
    const char* name;
    const void* p;
    bool needed;
  } arrays[] = {{"n_drafts", d_n_drafts, false}, {"drafts", d_drafts, max_drafts > 0}, {"p", d_p, true},
                {"q", d_q, false},               {"u", d_u, true},
                {"tokens", d_tokens, true},      {"accepted", d_accepted, true}};
  for (const auto& x : arrays) {
    if (&x - arrays < 5) {
      CHECK(check_place("tokens", d_tokens, 0, x.name, x.p, 0, false));
      CHECK(check_place("accepted", d_accepted, 0, x.name, x.p, 0, false));
    }
    if (!x.p && x.needed) return fail(SURGE_ERR_INVALID_ARGUMENT, "%s is NULL", x.name);
    if (!aligned(x.p, 4)) return fail(SURGE_ERR_INVALID_ARGUMENT, "%s must be 4-byte aligned", x.name);
  }
  CHECK(check_place("accepted", d_accepted, 0, "tokens", d_tokens, 0, false));
  if (ld_p < vocab || ld_p > kMostLength || (d_q && (ld_q < vocab || ld_q > kMostLength)))
    return fail(SURGE_ERR_INVALID_ARGUMENT, "row strides %lld and %lld of p and q, vocab=%d",
                (long long)ld_p, (long long)ld_q, vocab);
  const int64_t need = verify_workspace(n_seqs, vocab);
  if (need > 0) {
    CHECK(check_vector("workspace", d_workspace, true));
    if (workspace_bytes < need)
      return fail(SURGE_ERR_CAPACITY, "workspace of %lld bytes, %lld are needed",
                  (long long)workspace_bytes, (long long)need);
  }
  // A launch's threads: 1024 for every 32,768 tokens of a sequence.
  if (n_seqs * ((vocab + 32767) / 32768) > kMostThreads / 1024)
    return fail(SURGE_ERR_CAPACITY, "too many sequences and tokens for one call");
  int dev = 0, n_cus = 0;
  CHECK(current_device((hipStream_t)hip_stream, &dev, &n_cus));
  const VerifyDrafts a = {max_drafts, vocab, d_n_drafts, d_drafts,   d_p, d_q,
                          ld_p,       ld_q,  d_u,        d_tokens,   d_accepted, (double*)d_workspace};
  HIP_TRY(launch_verify_drafts(n_seqs, a, (hipStream_t)hip_stream));
  return SURGE_OK;
}

}  // extern "C"
