// SplitZip for MI355X (gfx950): the cache_ entry points of include/splitzip.h -- a KV cache in pages, quantised as it is
// written, and attention over it -- and the host side of their kernels.  The kernels live in the headers included below:
//   common.hpp      byte permutes and vector types shared with the codec
//   cache.hpp       where the words of a token are; writing, reading back, moving an accepted path
//   attention.hpp   attention of a step's rows, one token or a tree of drafted ones, over everything cached
#include <float.h>
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include <type_traits>

#include "splitzip.h"

namespace {

#include "common.hpp"
#include "cache.hpp"
#include "attention.hpp"

bool aligned16(uint64_t x) { return (x & 15u) == 0; }
bool aligned16(const void* p) { return aligned16((uint64_t)reinterpret_cast<uintptr_t>(p)); }
bool aligned(const void* p, unsigned n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1u)) == 0; }

int cu_count() {
  static int cached[64] = {0};
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return 256;
  if (!cached[dev]) {
    int n = 0;
    if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n <= 0) n = 256;
    cached[dev] = n;
  }
  return cached[dev];
}

int launched() { return hipGetLastError() == hipSuccess ? SPLITZIP_OK : SPLITZIP_ERR_HIP; }

constexpr uint64_t kMostTokens = 1u << 30;   // of a sequence: token numbers and the steps past them stay in 31 bits
constexpr uint64_t kMostRow = 1ull << 31;     // bytes of a row of the call's tensors: the place in one is a 32-bit offset
constexpr uint32_t kMostSeqs = 65535;        // a dimension of a grid
constexpr uint64_t kStreamed = 96ull << 20;   // bytes that a call moves (figures at the kernels)

int words_bytes(uint32_t dtype) { return dtype == SPLITZIP_BF16 ? 2 : 1; }

// a geometry's rules; the addresses of the words are looked at where a call has them
int check_cache(const splitzip_cache* c, bool pointers) {
  if (!c || c->dtype > SPLITZIP_FP8_E4M3 || c->reserved) return SPLITZIP_ERR_INVALID_ARG;
  if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256) return SPLITZIP_ERR_UNSUPPORTED;
  if (!c->kv_heads || !c->n_pages || c->page_tokens < 8 || c->page_tokens > kMostTokens) return SPLITZIP_ERR_INVALID_ARG;
  if (!aligned16(c->page_stride_bytes) || !aligned16(c->token_stride_bytes) || !aligned16(c->head_stride_bytes)) return SPLITZIP_ERR_INVALID_ARG;
  // eight tokens are a 32-bit offset, and so is a page
  if (c->token_stride_bytes > (1ull << 28) || c->page_stride_bytes >> 32 || c->scale_page_stride_bytes >> 32) return SPLITZIP_ERR_UNSUPPORTED;
  const uint64_t row = (uint64_t)c->head_dim * words_bytes(c->dtype);
  if (c->token_stride_bytes < row || c->head_stride_bytes < row) return SPLITZIP_ERR_INVALID_ARG;
  if (c->dtype != SPLITZIP_BF16 && (c->scale_page_stride_bytes & 7u || c->page_tokens & 7u)) return SPLITZIP_ERR_INVALID_ARG;
  if (!pointers) return SPLITZIP_OK;
  if (!c->d_k || !c->d_v || !aligned16(c->d_k) || !aligned16(c->d_v)) return SPLITZIP_ERR_INVALID_ARG;
  if (c->dtype != SPLITZIP_BF16 && (!c->d_k_scales || !c->d_v_scales || !aligned(c->d_k_scales, 8) || !aligned(c->d_v_scales, 8))) return SPLITZIP_ERR_INVALID_ARG;
  return SPLITZIP_OK;
}

int check_seqs(const splitzip_cache* c, const splitzip_seqs* q) {
  if (!q) return SPLITZIP_ERR_INVALID_ARG;
  if (q->n_seqs > kMostSeqs) return SPLITZIP_ERR_UNSUPPORTED;
  if (q->n_seqs && (!q->d_starts || !q->d_lens || !aligned(q->d_starts, 4) || !aligned(q->d_lens, 4) || !aligned(q->d_block_table, 4))) return SPLITZIP_ERR_INVALID_ARG;
  if (q->d_block_table) {
    if (!q->table_stride || (c->page_tokens & (c->page_tokens - 1))) return SPLITZIP_ERR_INVALID_ARG;
  } else if (q->n_seqs > c->n_pages || c->page_tokens & 7u) {
    return SPLITZIP_ERR_INVALID_ARG;
  }
  return SPLITZIP_OK;
}

Cache device_cache(const splitzip_cache* c, const splitzip_seqs* q) {
  Cache d;
  d.k = static_cast<uint8_t*>(c->d_k);
  d.v = static_cast<uint8_t*>(c->d_v);
  d.k_scales = c->dtype == SPLITZIP_BF16 ? nullptr : c->d_k_scales;
  d.v_scales = c->dtype == SPLITZIP_BF16 ? nullptr : c->d_v_scales;
  d.head_stride = c->head_stride_bytes;
  d.page_stride = (uint32_t)c->page_stride_bytes;
  d.token_stride = (uint32_t)c->token_stride_bytes;
  d.scale_page_stride = (uint32_t)c->scale_page_stride_bytes;
  d.page_shift = q->d_block_table ? 31u - (uint32_t)__builtin_clz(c->page_tokens) : 30u;
  d.page_tokens = c->page_tokens;
  d.last_page = c->n_pages - 1;
  d.heads = c->kv_heads;
  return d;
}

Seqs device_seqs(const splitzip_cache* c, const splitzip_seqs* q, uint32_t n_rows) {
  Seqs d;
  d.table = q->d_block_table;
  d.starts = q->d_starts;
  d.lens = q->d_lens;
  d.table_stride = q->table_stride;
  d.n_seqs = q->n_seqs;
  d.n_rows = n_rows;
  const uint64_t reach = q->d_block_table ? (uint64_t)q->table_stride * c->page_tokens : c->page_tokens;
  d.capacity = (uint32_t)(reach < kMostTokens ? reach : kMostTokens);
  return d;
}

bool rows_ok(const void* p, uint64_t stride, uint64_t elems) {
  return p && aligned16(p) && stride >= elems && stride % 8 == 0 && stride <= (1ull << 40);
}

// f<KIND, D>() for the cache's kind and width
template <template <int, int> class F, typename... A>
int by_kind(const splitzip_cache* c, A... args) {
#define SPLITZIP_KIND(K)                                          \
  if (c->dtype == K) {                                            \
    if (c->head_dim == 64) return F<K, 64>::run(args...);         \
    if (c->head_dim == 128) return F<K, 128>::run(args...);       \
    return F<K, 256>::run(args...);                               \
  }
  SPLITZIP_KIND(SPLITZIP_BF16)
  SPLITZIP_KIND(SPLITZIP_FP8_E5M2)
  SPLITZIP_KIND(SPLITZIP_FP8_E4M3)
#undef SPLITZIP_KIND
  return SPLITZIP_ERR_INVALID_ARG;
}

template <int KIND, int D>
struct Write {
  static int run(dim3 grid, bool stream, hipStream_t st, const RowsArgs* a) {
    if (stream) hipLaunchKernelGGL((cache_write_kernel<KIND, D, true>), grid, dim3(kThreads), 0, st, *a);
    else hipLaunchKernelGGL((cache_write_kernel<KIND, D, false>), grid, dim3(kThreads), 0, st, *a);
    return launched();
  }
};
template <int KIND, int D>
struct Read {
  static int run(dim3 grid, bool stream, hipStream_t st, const RowsArgs* a) {
    if (stream) hipLaunchKernelGGL((cache_read_kernel<KIND, D, true>), grid, dim3(kThreads), 0, st, *a);
    else hipLaunchKernelGGL((cache_read_kernel<KIND, D, false>), grid, dim3(kThreads), 0, st, *a);
    return launched();
  }
};

template <template <int, int> class F>
int rows_call(const splitzip_cache* c, const splitzip_seqs* q, void* d_k, uint64_t k_stride, void* d_v, uint64_t v_stride, uint32_t n_rows, void* stream) {
  int rc = check_cache(c, true);
  if (rc == SPLITZIP_OK) rc = check_seqs(c, q);
  if (rc != SPLITZIP_OK) return rc;
  const uint64_t elems = (uint64_t)c->kv_heads * c->head_dim;
  if (!q->n_seqs || !n_rows) return SPLITZIP_OK;
  if (n_rows > kMostTokens || elems * 2 > kMostRow) return SPLITZIP_ERR_UNSUPPORTED;
  if (!rows_ok(d_k, k_stride, elems) || !rows_ok(d_v, v_stride, elems)) return SPLITZIP_ERR_INVALID_ARG;
  RowsArgs a;
  a.cache = device_cache(c, q);
  a.seqs = device_seqs(c, q, n_rows);
  a.k = static_cast<uint8_t*>(d_k);
  a.v = static_cast<uint8_t*>(d_v);
  a.k_stride = 2 * k_stride;
  a.v_stride = 2 * v_stride;
  const uint64_t pairs = (uint64_t)(q->max_rows ? q->max_rows : 1) * c->kv_heads, per = (uint64_t)kAtOnce * kThreads / (c->head_dim / 8);
  uint64_t wgs = (pairs + per - 1) / per;
  const uint64_t most = (uint64_t)cu_count() * 32;
  if (wgs > most) wgs = most;
  const uint64_t bytes = 2 * n_rows * elems * (2 + words_bytes(c->dtype));
  return by_kind<F>(c, dim3((unsigned)wgs, q->n_seqs), bytes >= kStreamed, static_cast<hipStream_t>(stream), (const RowsArgs*)&a);
}

// How an attention call is cut: which kernel, the rows of a (sequence, head of the cache) into tiles, the tokens of all sequences
// into blocks and these into shares.
struct AttentionPlan {
  uint32_t waves, nt;   // waves 0: attention_tokens_kernel; else attention_rows_kernel with so many waves of 16 nt rows
  uint32_t heads_across, tile_rows, row_tiles, most_rows, kept;
  uint32_t shares, block_tokens, least_blocks;
  uint32_t wgs;
};
AttentionPlan plan_attention(const splitzip_cache* c, const splitzip_seqs* q, uint32_t q_heads) {
  AttentionPlan p;
  const uint64_t rows = (uint64_t)(q->max_rows ? q->max_rows : 1) * (q_heads / c->kv_heads);
  p.waves = 0;
  p.nt = 1;
  p.tile_rows = 16;
  // Two heads side by side and two waves for each.  us with one, two and four heads, sequences of eight heads of 128: BF16, one of 4000 tokens
  // 13.0, 14.3, 15.5, 16 of 4000 49.6, 51.0, 53.3, 64 of 200 14.3, 14.7, 23.1; E5M2 14.9, 13.1, 14.1, 35.9, 35.1, 38.2, 13.0, 12.0, 15.0;
  // 64 ragged ones of up to 8192 in shuffled pages 192, 181, 186.
  p.heads_across = rows > 16 || c->kv_heads % 2 ? 1u : 2u;
  const uint64_t longest = q->max_len < kMostTokens ? q->max_len : kMostTokens, tokens = q->n_seqs * longest;
  if (rows > 16) {
    // Four waves of 16 rows, three workgroups per CU, or eight of 32 rows, one: these read K and V less often, and have more to start and
    // to end with.  us the one way and the other, eight heads of 128, BF16: 8 sequences of 300 tokens and 128 rows 24.1 and 30.2, 2 of
    // 8000 and 256 rows 52 and 58, 8 of 4000 and 128 rows 62.5 and 56.8, 32 of 2000 and 128 rows 98 and 62; E5M2 24.0 and 29.2, 47.6 and 55.5, 55.3 and
    // 55.8, 82 and 62; 64 rows, 8 of 4000: 52.0 and 48.3, 43.4 and 46.7.  Rows of 256 elements leave a wave room for 16 rows only.
    const bool wide = rows > 64 && tokens * c->kv_heads >= 768ull * (uint64_t)cu_count();
    p.waves = wide || c->head_dim == 256 ? 8 : 4;
    p.nt = wide && c->head_dim != 256 ? 2 : 1;
    p.tile_rows = 16 * p.nt * p.waves;
  }
  const uint64_t tiles = (rows + p.tile_rows - 1) / p.tile_rows;
  p.row_tiles = (uint32_t)(tiles < 1024 ? tiles : 1024);
  p.most_rows = (uint32_t)(rows < (uint64_t)p.row_tiles * p.tile_rows ? rows : (uint64_t)p.row_tiles * p.tile_rows);
  p.kept = (uint32_t)(rows < p.tile_rows ? rows : p.tile_rows);
  // as many workgroups as the chip holds at a time: two with 64 KB of LDS per CU, one with 128 KB or eight waves, three with 32 KB
  const bool one_per_cu = p.waves == 8 || (p.waves == 0 && c->dtype == SPLITZIP_BF16 && c->head_dim == 256);
  const uint64_t groups = (uint64_t)(c->kv_heads / p.heads_across) * p.row_tiles, slots = (uint64_t)cu_count() * (one_per_cu ? 1 : p.waves ? 3 : 2);
  uint64_t shares = (slots + groups - 1) / groups;
  // a block: what the waves of a head stage at a time
  const uint32_t staged = p.waves ? p.waves * 1024u / c->head_dim : 8192u / (c->head_dim * words_bytes(c->dtype));
  p.block_tokens = p.waves ? staged : (staged < 32 ? 32 : staged) * (kWaves / p.heads_across);
  // (a sum of blocks is kept in 32 bits)
  const uint64_t most = (uint64_t)q->n_seqs * (q->d_block_table ? (uint64_t)q->table_stride * c->page_tokens : c->page_tokens);
  while (most / p.block_tokens + q->n_seqs > (1ull << 31) && p.block_tokens < (1u << 30)) p.block_tokens *= 2;
  // Rows of a tree take at least a sixteenth of all tokens, 64 to 256 of them, since more rows are more to join: us with 64, 128, 256 and 512
  // tokens, 52 rows of 8 heads, one sequence of 1000 tokens 14.4, 15.3, 16.3, 20.8, four 19.6, 16.9, 17.0, 21.4, one of 4000 22.3, 19.4, 17.7, 22.3.
  const uint64_t least = tokens / 16 < 64 ? 64 : tokens / 16 > 256 ? 256 : tokens / 16;
  p.least_blocks = p.waves && p.block_tokens < least ? (uint32_t)(least / p.block_tokens) : 1;
  // Short sequences are not cut: parts of them would gain less than the launch that joins them costs (5 us, more for many rows).  The longer, the more
  // there is to do side by side anyway.  us cut and not, E5M2, heads of 64: a sequence of 468 tokens 12.0 and 11.0, of 625 12.0 and 13.2, 64 of
  // 1000 32.7 and 28.3; of 128: a sequence of 234 11.6 and 10.4, 8 of 468 12.6 and 15.0, 52 rows 8 of 400 19.4 and 15.7, 8 of 800 21.6
  // and 24.5, 32 of 1000 46 and 34, 256 rows 4 of 300 27 and 14; of 256: a sequence of 117 13.4 and 11.9, 8 of 234 15.5 and 16.3, 256 rows 4 of 300 46 and 22.
  const uint64_t units = (uint64_t)q->n_seqs * c->kv_heads * ((rows + 15) / 16);
  if (longest * c->head_dim <= 32768 + 96 * (units < 1024 ? units : 1024)) {   // every sequence is a block
    p.block_tokens = (uint32_t)kMostTokens;
    p.least_blocks = 1;
  }
  const uint64_t blocks = q->n_seqs * (longest ? (longest + p.block_tokens - 1) / p.block_tokens : 1);   // by what the call says
  if (shares > (blocks + p.least_blocks - 1) / p.least_blocks) shares = (blocks + p.least_blocks - 1) / p.least_blocks;
  if (shares < 1) shares = 1;
  p.shares = (uint32_t)shares;
  p.wgs = (uint32_t)((shares * (c->kv_heads / p.heads_across) + 7) / 8 * 8 * p.row_tiles);
  return p;
}

template <int KIND, int D>
struct Attend {
  template <int W, int NT, bool PLAIN>
  static void rows(dim3 grid, hipStream_t st, const AttentionArgs* a) {
    hipLaunchKernelGGL((attention_rows_kernel<KIND, D, W, NT, PLAIN>), grid, dim3(64 * W), 0, st, *a);
  }
  template <bool PLAIN>
  static void any(dim3 grid, uint32_t waves, hipStream_t st, const AttentionArgs* a) {
    if (!waves) hipLaunchKernelGGL((attention_tokens_kernel<KIND, D, PLAIN>), grid, dim3(kThreads), 0, st, *a);
    else if constexpr (D == 256) rows<8, 1, PLAIN>(grid, st, a);
    else waves == 4 ? rows<4, 1, PLAIN>(grid, st, a) : rows<8, 2, PLAIN>(grid, st, a);
  }
  static int run(dim3 grid, uint32_t waves, hipStream_t st, const AttentionArgs* a) {
    // (a scale of 0 times an infinity that is not seen would be a NaN: not plain)
    if (a->softcap == 0.0f && !a->slopes && a->scale > 0.0f) any<true>(grid, waves, st, a);
    else any<false>(grid, waves, st, a);
    return launched();
  }
};

uint64_t parts_of(const AttentionPlan& p) { return (uint64_t)p.wgs * 2 * p.heads_across * p.kept; }
// whether a sequence may be taken by several workgroups
bool cuts(const AttentionPlan& p) { return p.shares > 1 && p.block_tokens < kMostTokens; }
uint64_t workspace_of(const AttentionPlan& p, const splitzip_cache* c) { return !cuts(p) ? 0 : parts_of(p) * (c->head_dim + 2) * sizeof(float); }

}  // namespace

extern "C" {

int splitzip_cache_write(const splitzip_cache* cache, const splitzip_seqs* seqs, const void* d_k, uint64_t k_row_stride, const void* d_v,
                         uint64_t v_row_stride, uint32_t n_rows, void* stream) {
  return rows_call<Write>(cache, seqs, const_cast<void*>(d_k), k_row_stride, const_cast<void*>(d_v), v_row_stride, n_rows, stream);
}

int splitzip_cache_read(const splitzip_cache* cache, const splitzip_seqs* seqs, void* d_k, uint64_t k_row_stride, void* d_v, uint64_t v_row_stride,
                        uint32_t n_rows, void* stream) {
  return rows_call<Read>(cache, seqs, d_k, k_row_stride, d_v, v_row_stride, n_rows, stream);
}

size_t splitzip_attention_workspace_bytes(const splitzip_cache* cache, const splitzip_seqs* seqs, uint32_t n_rows, uint32_t q_heads) {
  if (check_cache(cache, false) != SPLITZIP_OK || check_seqs(cache, seqs) != SPLITZIP_OK || !q_heads || q_heads % cache->kv_heads) return 0;
  return n_rows ? (size_t)workspace_of(plan_attention(cache, seqs, q_heads), cache) : 0;
}

int splitzip_cache_attention(const splitzip_cache* cache, const splitzip_seqs* seqs, const splitzip_attention* how, const void* d_q,
                             uint64_t q_row_stride, void* d_out, uint64_t out_row_stride, float* d_lse, uint32_t n_rows, uint32_t q_heads,
                             void* d_workspace, size_t workspace_bytes, void* stream) {
  int rc = check_cache(cache, true);
  if (rc == SPLITZIP_OK) rc = check_seqs(cache, seqs);
  if (rc != SPLITZIP_OK) return rc;
  if (!how || !q_heads || q_heads % cache->kv_heads || !(how->softcap == 0.0f || (how->softcap >= FLT_MIN && how->softcap <= FLT_MAX)) || how->reserved) return SPLITZIP_ERR_INVALID_ARG;
  if (!aligned(how->d_slopes, 4) || !aligned(how->d_tree, 8) || !aligned(how->d_positions, 4) || (how->d_tree && !how->tree_words)) return SPLITZIP_ERR_INVALID_ARG;
  if (!seqs->n_seqs || !n_rows) return SPLITZIP_OK;
  const uint64_t elems = (uint64_t)q_heads * cache->head_dim;
  if (n_rows > kMostTokens || elems * 2 > kMostRow) return SPLITZIP_ERR_UNSUPPORTED;
  const AttentionPlan p = plan_attention(cache, seqs, q_heads);
  const uint64_t need = workspace_of(p, cache);
  if (workspace_bytes < need) return SPLITZIP_ERR_CAPACITY;
  if (need && (!d_workspace || !aligned16(d_workspace))) return SPLITZIP_ERR_INVALID_ARG;
  if (!rows_ok(d_q, q_row_stride, elems) || !rows_ok(d_out, out_row_stride, elems) || !aligned(d_lse, 4)) return SPLITZIP_ERR_INVALID_ARG;
  AttentionArgs a;
  a.cache = device_cache(cache, seqs);
  a.seqs = device_seqs(cache, seqs, n_rows);
  a.q = static_cast<const uint8_t*>(d_q);
  a.out = static_cast<uint8_t*>(d_out);
  a.lse = d_lse;
  a.q_stride = 2 * q_row_stride;
  a.out_stride = 2 * out_row_stride;
  a.slopes = how->d_slopes;
  a.tree = how->d_tree;
  a.positions = how->d_positions;
  a.part_out = static_cast<float*>(d_workspace);
  a.part_stat = a.part_out + parts_of(p) * cache->head_dim;
  a.scale = how->scale < 0.0f ? -how->scale : how->scale;
  a.flip_q = how->scale < 0.0f ? 0x80008000u : 0u;
  a.softcap = how->softcap;
  a.tree_words = how->tree_words;
  a.window = how->window;
  a.group = q_heads / cache->kv_heads;
  a.heads_across = p.heads_across;
  a.tile_rows = p.tile_rows;
  a.row_tiles = p.row_tiles;
  a.most_rows = p.most_rows;
  a.kept = p.kept;
  a.shares = p.shares;
  a.block_tokens = p.block_tokens;
  a.least_blocks = p.least_blocks;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  rc = by_kind<Attend>(cache, dim3(p.wgs), p.waves, st, (const AttentionArgs*)&a);
  if (rc != SPLITZIP_OK || !cuts(p)) return rc;
  const uint64_t outs = (uint64_t)(seqs->max_rows ? seqs->max_rows : 1) * q_heads;
  // a workgroup for each row and head, or, since it takes 256 threads' worth of rows at a time where parts are few, for so many of them
  const uint64_t at_a_time = 4 * kThreads / cache->head_dim, few = (outs + at_a_time - 1) / at_a_time, held = (uint64_t)cu_count() * 8 / seqs->n_seqs + 1;
  const uint64_t each = outs < (uint64_t)cu_count() / seqs->n_seqs ? outs : (uint64_t)cu_count() / seqs->n_seqs;
  const uint64_t wgs = few < held ? few : held;
  const dim3 grid((unsigned)(wgs > each ? wgs : each), seqs->n_seqs);
  if (cache->head_dim == 64) hipLaunchKernelGGL(attention_join_kernel<64>, grid, dim3(kThreads), 0, st, a);
  else if (cache->head_dim == 128) hipLaunchKernelGGL(attention_join_kernel<128>, grid, dim3(kThreads), 0, st, a);
  else hipLaunchKernelGGL(attention_join_kernel<256>, grid, dim3(kThreads), 0, st, a);
  return launched();
}

int splitzip_cache_move(const splitzip_cache* caches, uint32_t n_caches, const splitzip_seqs* seqs, const int32_t* d_path, uint32_t path_stride,
                        uint32_t n_rows, void* stream) {
  if (!n_caches) return SPLITZIP_OK;
  if (!caches) return SPLITZIP_ERR_INVALID_ARG;
  for (uint32_t k = 0; k < n_caches; ++k) {
    const splitzip_cache &c = caches[k], &f = caches[0];
    const int rc = check_cache(&c, true);
    if (rc != SPLITZIP_OK) return rc;
    if (c.dtype != f.dtype || c.kv_heads != f.kv_heads || c.head_dim != f.head_dim || c.page_tokens != f.page_tokens || c.n_pages != f.n_pages ||
        c.page_stride_bytes != f.page_stride_bytes || c.token_stride_bytes != f.token_stride_bytes || c.head_stride_bytes != f.head_stride_bytes ||
        (c.dtype != SPLITZIP_BF16 && c.scale_page_stride_bytes != f.scale_page_stride_bytes))
      return SPLITZIP_ERR_INVALID_ARG;
  }
  const int rc = check_seqs(caches, seqs);
  if (rc != SPLITZIP_OK) return rc;
  if (!seqs->n_seqs || !path_stride || !n_rows) return SPLITZIP_OK;
  if (!d_path || !aligned(d_path, 4)) return SPLITZIP_ERR_INVALID_ARG;
  if (n_rows > kMostTokens || (uint64_t)caches->kv_heads * caches->head_dim > (1u << 28)) return SPLITZIP_ERR_UNSUPPORTED;
  MoveArgs a;
  a.cache = device_cache(caches, seqs);
  a.seqs = device_seqs(caches, seqs, n_rows);
  a.path = d_path;
  a.path_stride = path_stride;
  a.row_bytes = caches->head_dim * (uint32_t)words_bytes(caches->dtype);
  for (uint32_t at = 0; at < n_caches; at += kMoveMax) {
    const uint32_t n = n_caches - at < kMoveMax ? n_caches - at : kMoveMax;
    for (uint32_t k = 0; k < n; ++k) {
      const Cache d = device_cache(caches + at + k, seqs);
      a.at[k].k = d.k;
      a.at[k].v = d.v;
      a.at[k].k_scales = d.k_scales;
      a.at[k].v_scales = d.v_scales;
    }
    for (uint32_t k = n; k < kMoveMax; ++k) a.at[k].k = a.at[k].v = a.at[k].k_scales = a.at[k].v_scales = nullptr;
    hipLaunchKernelGGL(cache_move_kernel, dim3(seqs->n_seqs, n), dim3(kThreads), 0, static_cast<hipStream_t>(stream), a);
    const int rl = launched();
    if (rl != SPLITZIP_OK) return rl;
  }
  return SPLITZIP_OK;
}

}  // extern "C"
