// SplitZip for MI355X: a KV cache in pages -- where its words live, and the kernels that write tokens into it, read them back and
// move them.  Part of the single translation unit cache.hip (included inside its anonymous namespace).
//
// An FP8 cache keeps one scale per token and head, a power of two 2^e stored as the byte e + 127: the least e in
// [-127, 127] with max |x| <= 1.75 * 2^(X + e), where 1.75 * 2^X is the format's largest finite word (X = 15 for E5M2, 8 for
// E4M3).  The words are a floating format, so a power of two loses them nothing against any other scale but what it moves into
// their subnormal range; x 2^-e is exact, so a word is rounded once; and the words' exponents lie in the same place in
// every tensor, which is what the codec's codebooks count on.  Sums are not taken anywhere here: a largest magnitude and
// products with powers of two are exact in 32 bits.
#ifndef SPLITZIP_CACHE_HPP
#define SPLITZIP_CACHE_HPP

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kTopE5m2 = 15, kTopE4m3 = 8;

// the words of K and V and their scales; a page is where the table says, or, without a table, sequence s is page s
struct Cache {
  uint8_t *k, *v;
  uint8_t *k_scales, *v_scales;
  uint64_t head_stride;                                 // bytes
  uint32_t page_stride, token_stride, scale_page_stride;   // bytes: a product with a 32-bit number is one instruction
  uint32_t page_shift;   // log2 of the tokens per page, at least 3: eight tokens in a row from a multiple of eight share a page
  uint32_t page_tokens;
  uint32_t last_page, heads;
};

// sequences: rows [starts[s], starts[s + 1]) of this call's tensors are the last tokens of the lens[s] that s has in the cache
struct Seqs {
  const uint32_t* table;
  const int32_t *starts, *lens;
  uint32_t table_stride, n_seqs, n_rows;
  uint32_t capacity;   // tokens that a row of the table reaches
};

struct Seq {
  int start, rows, len, base;   // base: tokens in front of this call's rows (below zero where a length is shorter than the rows)
};
// nothing that starts and lens say leads outside the call's tensors or the table
__device__ inline Seq seq_at(const Seqs& q, uint32_t s) {
  Seq r;
  const int a = q.starts[s], b = q.starts[s + 1], n = q.lens[s];
  r.start = min(max(a, 0), (int)q.n_rows);
  r.rows = max(min(b, (int)q.n_rows), r.start) - r.start;   // (the difference is taken last: b may be any number)
  r.len = min(max(n, 0), (int)q.capacity);
  r.base = r.len - r.rows;
  return r;
}

// where a sequence's tokens are
struct Pages {
  const uint32_t* row;     // of the table, or null
  uint32_t seq, shift, mask, last;
  __device__ Pages() {}
  __device__ Pages(const Cache& c, const Seqs& q, uint32_t s)
      : row(q.table ? q.table + (uint64_t)s * q.table_stride : nullptr), seq(s), shift(c.page_shift), mask(q.table ? c.page_tokens - 1 : ~0u), last(c.last_page) {}
  // of token t, below the sequence's length: the page in the pool (a bad table entry never leaves it), the place in the page
  __device__ uint32_t page(uint32_t t) const { return clamped(entry(t)); }
  // the same in two steps: a loop that asks for the entry well ahead must not touch it before it is needed, or it waits for
  // everything that it has asked for before
  __device__ uint32_t entry(uint32_t t) const { return row ? row[t >> shift] : seq; }
  __device__ uint32_t clamped(uint32_t entry) const { return min(entry, last); }
  __device__ uint32_t place(uint32_t t) const { return t & mask; }
};
// byte of a token's words, heads apart; the same offset in K and V
__device__ inline uint64_t token_offset(const Cache& c, uint32_t page, uint32_t place) {
  return (uint64_t)page * c.page_stride + (uint64_t)place * c.token_stride;
}
// byte of its scale: [heads][tokens of a page], so that the scales of eight tokens of a head are one load
__device__ inline uint64_t scale_offset(const Cache& c, uint32_t page, uint32_t place, uint32_t head) {
  return (uint64_t)page * c.scale_page_stride + (uint64_t)head * c.page_tokens + place;
}

// 16 bytes per lane from memory straight into LDS: the wave's lanes one behind the other from `to` on, which is the wave's.  They are
// there when memory_arrived says so.  Streamed: nothing else reads them.
__device__ inline void load_to_lds(const uint8_t* from, uint8_t* to) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from, (__attribute__((address_space(3))) void*)to, 16, 0, kStream);
}
__device__ inline void memory_arrived() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
__device__ inline void lds_read() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

struct RowsArgs {
  Cache cache;
  Seqs seqs;
  uint8_t *k, *v;          // the call's tensors of BF16 rows
  uint64_t k_stride, v_stride;   // bytes from row to row
};

// waits for the wave's own accesses to LDS, not for its loads from memory, which stay on their way
__device__ inline void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// largest finite magnitude of eight BF16 words, as bits (which order as the magnitudes do)
__device__ inline uint32_t largest8(const u32x4& w) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t lo = w[i] & 0x7fffu, hi = (w[i] >> 16) & 0x7fffu;
    m = max(m, lo < 0x7f80u ? lo : 0u);
    m = max(m, hi < 0x7f80u ? hi : 0u);
  }
  return m;
}

// the scale byte for a largest magnitude of these BF16 bits
template <int TOP>
__device__ inline int scale_byte(uint32_t bits) {
  const uint32_t f = bits << 16;
  int e = (int)(f >> 23) - 127;
  uint32_t mant = f & 0x7fffffu;
  if (!(f >> 23)) {   // a subnormal: shifted up to its first bit
    const int up = __builtin_clz(mant | 1u) - 8;
    e = -126 - up;
    mant = (mant << up) & 0x7fffffu;
  }
  e = e - TOP + (mant > 0x600000u ? 1 : 0);
  return bits && e > -127 ? e + 127 : 0;
}

// 8 BF16 words times 2^(127 - byte), rounded to FP8: 8 bytes.  2^(127 - byte) as two factors, each a normal number.
template <int KIND>
__device__ inline u32x2 to_fp8(const u32x4& w, int byte) {
  const int up = 127 - byte, half = up / 2;
  const float a = __uint_as_float((uint32_t)(127 + half) << 23), b = __uint_as_float((uint32_t)(127 + up - half) << 23);
  u32x2 out;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const float x0 = __uint_as_float(w[2 * i] << 16) * a * b, x1 = __uint_as_float(w[2 * i] & 0xffff0000u) * a * b;
    const float x2 = __uint_as_float(w[2 * i + 1] << 16) * a * b, x3 = __uint_as_float(w[2 * i + 1] & 0xffff0000u) * a * b;
    int d = 0;
    if constexpr (KIND == SPLITZIP_FP8_E5M2) {
      d = __builtin_amdgcn_cvt_pk_bf8_f32(x0, x1, d, false);
      d = __builtin_amdgcn_cvt_pk_bf8_f32(x2, x3, d, true);
    } else {
      d = __builtin_amdgcn_cvt_pk_fp8_f32(x0, x1, d, false);
      d = __builtin_amdgcn_cvt_pk_fp8_f32(x2, x3, d, true);
    }
    out[i] = (uint32_t)d;
  }
  return out;
}

// The words of a pair of bytes (the low or the high two of a register) times 2^(byte - 127), rounded to BF16.  The instruction takes the
// power from the exponent field of a number in 32 bits (the field 0 stands for 2^-127): the byte, shifted there.  A word has four
// significant bits at most, so only results below BF16's normal numbers are rounded, once, and those at 2^128 become infinite.
template <int KIND, bool HIGH>
__device__ inline uint32_t fp8_pair_to_bf16(uint32_t w, uint32_t byte) {
  bf16x2 r;
  if constexpr (KIND == SPLITZIP_FP8_E5M2) r = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(w, __uint_as_float(byte << 23), HIGH);
  else r = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, __uint_as_float(byte << 23), HIGH);
  return __builtin_bit_cast(uint32_t, r);
}

// nearest BF16, ties to even
__device__ inline uint32_t bf16_pair(float lo, float hi) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{lo, hi}, bf16x2));
}

// 8 FP8 words times 2^(byte - 127) as BF16
template <int KIND>
__device__ inline u32x4 from_fp8(const u32x2& w, uint32_t byte) {
  return u32x4{fp8_pair_to_bf16<KIND, false>(w[0], byte), fp8_pair_to_bf16<KIND, true>(w[0], byte), fp8_pair_to_bf16<KIND, false>(w[1], byte),
               fp8_pair_to_bf16<KIND, true>(w[1], byte)};
}

// Rows into the cache, and back.  A row of a head is taken by D / 8 lanes, eight elements each; a workgroup belongs to one
// sequence (blockIdx.y) and takes kAtOnce (row, head) pairs per lane at a time, K and V of a pair together: all of their words are asked for before
// the first is used.
//
// Bound by memory.  Calls that move more than the last-level cache can be of use for (96 MB of its 256) read and, back out of
// the cache, write past it.  us a call, ordinary and streamed, five sets of tensors in turn, so that nothing of a call is in a cache (in
// brackets two sets, where it may be):
//                        7126 tokens of 8 x 128         16 384              32 768               65 536
//   write E4M3                                       (19.4 / 20.8)          40.0 / 35.1       (79.8 / 69.6)
//   read E5M2                                         22.5 / 20.1           41.2 / 37.4       (79.2 / 72.8)
//   read BF16                  12.4 / 12.3                                  52.9 / 47.5       (104 / 92)
// (32 768 tokens written: 201 MB at 5.7 TB/s, read 5.4, BF16 5.65; a plain copy of that mix of reads and writes 5.4 to 5.7).  One pair at a time
// instead of two 37.5 and 46.6 (read, E5M2 and BF16) and 38.1 and 42.5 (written) where two take 36.0 and 41.4.
constexpr int kAtOnce = 2;
template <bool STREAM, typename T>
__device__ inline T ld_row(const uint8_t* p) {
  if constexpr (STREAM) return ld_stream(reinterpret_cast<const T*>(p));
  else return *reinterpret_cast<const T*>(p);
}
template <int D>
struct Pairs {
  static constexpr uint32_t kLanes = D / 8, kOfWg = kThreads / kLanes, kStepPairs = kOfWg * kAtOnce;
  Seq s;
  Pages pages;
  uint32_t n;          // (row, head) pairs of the sequence
  uint32_t row[kAtOnce], heads[kAtOnce];   // of the call's tensors, of the cache
  int token[kAtOnce];  // below zero: nowhere
  __device__ Pairs(const RowsArgs& a) : s(seq_at(a.seqs, blockIdx.y)), pages(a.cache, a.seqs, blockIdx.y), n((uint32_t)s.rows * a.cache.heads) {}
  // pair j of those from p0 on; false if there is none (then it is the last one once more: what is loaded for it is there, and no load
  // stands behind a condition)
  __device__ bool at(const RowsArgs& a, uint32_t p0, int j) {
    const uint32_t p = p0 + (uint32_t)j * kOfWg + threadIdx.x / kLanes, q = min(p, n - 1), i = q / a.cache.heads;
    row[j] = (uint32_t)s.start + i;
    heads[j] = q - i * a.cache.heads;
    token[j] = s.base + (int)i;
    return p < n;
  }
};

template <int KIND, int D, bool STREAM>
__global__ void __launch_bounds__(kThreads) cache_write_kernel(RowsArgs a) {
  Pairs<D> p(a);
  const uint32_t lane = threadIdx.x % Pairs<D>::kLanes;
  for (uint32_t p0 = blockIdx.x * Pairs<D>::kStepPairs; p0 < p.n; p0 += gridDim.x * Pairs<D>::kStepPairs) {
    bool have[kAtOnce];
    u32x4 k[kAtOnce], v[kAtOnce];
    uint32_t page[kAtOnce];
#pragma unroll
    for (int j = 0; j < kAtOnce; ++j) {
      have[j] = p.at(a, p0, j) && p.token[j] >= 0;
      const uint32_t at = 2 * (p.heads[j] * D + lane * 8);
      page[j] = p.pages.entry((uint32_t)max(p.token[j], 0));
      k[j] = ld_row<STREAM, u32x4>(a.k + p.row[j] * a.k_stride + at);
      v[j] = ld_row<STREAM, u32x4>(a.v + p.row[j] * a.v_stride + at);
    }
#pragma unroll
    for (int j = 0; j < kAtOnce; ++j) {
      if (!have[j]) continue;
      const uint32_t in = p.pages.clamped(page[j]), place = p.pages.place((uint32_t)p.token[j]);
      const uint64_t word = token_offset(a.cache, in, place) + p.heads[j] * a.cache.head_stride;
      if constexpr (KIND == SPLITZIP_BF16) {
        *reinterpret_cast<u32x4*>(a.cache.k + word + lane * 16) = k[j];
        *reinterpret_cast<u32x4*>(a.cache.v + word + lane * 16) = v[j];
      } else {
        uint32_t mk = largest8(k[j]), mv = largest8(v[j]);
#pragma unroll
        for (int o = Pairs<D>::kLanes / 2; o > 0; o /= 2) {
          mk = max(mk, (uint32_t)__shfl_xor((int)mk, o));
          mv = max(mv, (uint32_t)__shfl_xor((int)mv, o));
        }
        constexpr int kTop = KIND == SPLITZIP_FP8_E5M2 ? kTopE5m2 : kTopE4m3;
        const int bk = scale_byte<kTop>(mk), bv = scale_byte<kTop>(mv);
        *reinterpret_cast<u32x2*>(a.cache.k + word + lane * 8) = to_fp8<KIND>(k[j], bk);
        *reinterpret_cast<u32x2*>(a.cache.v + word + lane * 8) = to_fp8<KIND>(v[j], bv);
        if (lane == 0) {
          const uint64_t scale = scale_offset(a.cache, in, place, p.heads[j]);
          a.cache.k_scales[scale] = (uint8_t)bk;
          a.cache.v_scales[scale] = (uint8_t)bv;
        }
      }
    }
  }
}

template <int KIND, int D, bool STREAM>
__global__ void __launch_bounds__(kThreads) cache_read_kernel(RowsArgs a) {
  constexpr int ES = KIND == SPLITZIP_BF16 ? 2 : 1;
  typedef typename std::conditional<ES == 2, u32x4, u32x2>::type Words;
  Pairs<D> p(a);
  const uint32_t lane = threadIdx.x % Pairs<D>::kLanes;
  for (uint32_t p0 = blockIdx.x * Pairs<D>::kStepPairs; p0 < p.n; p0 += gridDim.x * Pairs<D>::kStepPairs) {
    bool have[kAtOnce];
    Words k[kAtOnce], v[kAtOnce];
    uint32_t page[kAtOnce], bk[kAtOnce], bv[kAtOnce];
#pragma unroll
    for (int j = 0; j < kAtOnce; ++j) {
      have[j] = p.at(a, p0, j);
      page[j] = p.pages.entry((uint32_t)max(p.token[j], 0));
    }
#pragma unroll
    for (int j = 0; j < kAtOnce; ++j) {
      const uint32_t in = p.pages.clamped(page[j]), place = p.pages.place((uint32_t)max(p.token[j], 0));
      const uint64_t word = token_offset(a.cache, in, place) + p.heads[j] * a.cache.head_stride + lane * 8 * ES;
      k[j] = ld_row<STREAM, Words>(a.cache.k + word);
      v[j] = ld_row<STREAM, Words>(a.cache.v + word);
      if constexpr (ES == 1) {
        const uint64_t scale = scale_offset(a.cache, in, place, p.heads[j]);
        bk[j] = a.cache.k_scales[scale];
        bv[j] = a.cache.v_scales[scale];
      }
    }
#pragma unroll
    for (int j = 0; j < kAtOnce; ++j) {
      if (!have[j]) continue;
      const uint32_t at = 2 * (p.heads[j] * D + lane * 8);
      u32x4 ko, vo;
      if constexpr (ES == 2) {
        ko = k[j];
        vo = v[j];
      } else {
        ko = from_fp8<KIND>(k[j], bk[j]);
        vo = from_fp8<KIND>(v[j], bv[j]);
      }
      if (p.token[j] < 0) ko = vo = u32x4{0, 0, 0, 0};   // a row in front of the sequence's first token
      u32x4 *const k_to = reinterpret_cast<u32x4*>(a.k + p.row[j] * a.k_stride + at), *const v_to = reinterpret_cast<u32x4*>(a.v + p.row[j] * a.v_stride + at);
      if constexpr (STREAM) {
        st_stream(k_to, ko);
        st_stream(v_to, vo);
      } else {
        *k_to = ko;
        *v_to = vo;
      }
    }
  }
}

// The accepted path of a tree of drafted tokens: token base + path[i] becomes token base + i.  A path ascends strictly, so
// path[i] >= i, and token i is not among the sources behind the i-th: a thread that reads and writes its 16 bytes (or its scale) of
// the tokens in the path's order, or reads those of several before it writes them, never reads what it has written.
// Entries that do not ascend, or are no rows of the call, end the path.
constexpr uint32_t kMoveMax = 64;   // caches of a launch
struct MoveArgs {
  Cache cache;             // the geometry all of them share
  Seqs seqs;
  const int32_t* path;
  uint32_t path_stride, row_bytes;   // entries per sequence; bytes of a token and head
  struct { uint8_t *k, *v, *k_scales, *v_scales; } at[kMoveMax];
};
// Bound by latency: the starts, the path, the table and the tokens are asked for one behind the other, each of them once for 64 entries of
// the path (a lane each) or eight tokens (a register each).  48 paths of up to 6 tokens in 32 layers of E5M2 (25 MB): 8.6 us.
__global__ void __launch_bounds__(kThreads) cache_move_kernel(MoveArgs a) {
  constexpr uint32_t kHeld = 8;
  const uint32_t lane = threadIdx.x % 64, first_piece = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x - lane));   // a wave's
  const int32_t* path = a.path + (uint64_t)blockIdx.x * a.path_stride;
  const Seq s = seq_at(a.seqs, blockIdx.x);
  const Pages at_pages(a.cache, a.seqs, blockIdx.x);
  const auto& at = a.at[blockIdx.y];
  const uint32_t per_head = a.row_bytes / 16, pieces = per_head * a.cache.heads, each = pieces + (at.k_scales ? a.cache.heads : 0);   // of K, and of V
  int before = -1;
  for (uint32_t i0 = 0; i0 < a.path_stride; i0 += 64) {
    // the entries of the path that are part of it, a lane each
    const uint32_t i = i0 + lane;
    const int from = i < a.path_stride ? path[i] : -1, last = (int)lane_before((uint32_t)from, (uint32_t)before);
    const uint64_t ends = ~__ballot(from > last && from < s.rows);
    const uint32_t n = ends ? (uint32_t)__builtin_ctzll(ends) : 64;
    const uint32_t t = (uint32_t)max(s.base + from, 0), to = (uint32_t)max(s.base + (int)i, 0);
    const bool moves = lane < n && from != (int)i && s.base + (int)i >= 0;
    uint32_t p0 = 0, p1 = 0;
    if (moves) {
      p0 = at_pages.entry(t);
      p1 = at_pages.entry(to);
    }
    p0 = at_pages.clamped(p0);
    p1 = at_pages.clamped(p1);
    const uint32_t l0 = at_pages.place(t), l1 = at_pages.place(to);
    // The lanes hold the path's entries, so all 64 of them go through the pieces, also those that have no piece of their own any more:
    // they take the last one, and do not write it.
    const uint64_t moving = __ballot(moves);
    for (uint32_t u0 = first_piece; u0 < 2 * each; u0 += kThreads) {
      const bool live = u0 + lane < 2 * each;
      const uint32_t u = min(u0 + lane, 2 * each - 1);
      const bool of_v = u >= each, is_word = u - (of_v ? each : 0) < pieces;
      const uint32_t w = u - (of_v ? each : 0), head = is_word ? w / per_head : w - pieces;
      uint8_t* const words = (of_v ? at.v : at.k) + head * a.cache.head_stride + (is_word ? w - head * per_head : 0) * 16;
      uint8_t* const scales = of_v ? at.v_scales : at.k_scales;
      for (uint64_t left = moving; left;) {
        u32x4 x[kHeld];
        uint64_t dst[kHeld];
        uint32_t held = 0;
#pragma unroll
        for (uint32_t j = 0; j < kHeld; ++j) {
          if (!left) break;
          const int l = __builtin_ctzll(left);
          left &= left - 1;
          const uint32_t sp = (uint32_t)__builtin_amdgcn_readlane((int)p0, l), sl = (uint32_t)__builtin_amdgcn_readlane((int)l0, l);
          const uint32_t dp = (uint32_t)__builtin_amdgcn_readlane((int)p1, l), dl = (uint32_t)__builtin_amdgcn_readlane((int)l1, l);
          if (is_word) {
            x[j] = *reinterpret_cast<const u32x4*>(words + token_offset(a.cache, sp, sl));
            dst[j] = token_offset(a.cache, dp, dl);
          } else {
            x[j][0] = scales[scale_offset(a.cache, sp, sl, head)];
            dst[j] = scale_offset(a.cache, dp, dl, head);
          }
          held = j + 1;
        }
#pragma unroll
        for (uint32_t j = 0; j < kHeld; ++j) {
          if (j >= held) break;
          if (!live) continue;
          if (is_word) *reinterpret_cast<u32x4*>(words + dst[j]) = x[j];
          else scales[dst[j]] = (uint8_t)x[j][0];
        }
      }
    }
    if (n < 64) break;
    before = __builtin_amdgcn_readlane(from, 63);
  }
}

#endif  // SPLITZIP_CACHE_HPP
