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
  r.rows = max(min(b, (int)q.n_rows) - r.start, 0);
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
// sequence (blockIdx.y) and takes its (row, head) pairs in turn, K and V of a pair together.
template <int KIND, int D>
__global__ void __launch_bounds__(kThreads) cache_write_kernel(RowsArgs a) {
  constexpr int kLanes = D / 8, kPairs = kThreads / kLanes;
  const Seq s = seq_at(a.seqs, blockIdx.y);
  const Pages at_pages(a.cache, a.seqs, blockIdx.y);
  const uint32_t lane = threadIdx.x % kLanes, pairs = (uint32_t)s.rows * a.cache.heads;
  for (uint32_t p = blockIdx.x * kPairs + threadIdx.x / kLanes; p < pairs; p += gridDim.x * kPairs) {
    const uint32_t i = p / a.cache.heads, head = p - i * a.cache.heads;
    const int t = s.base + (int)i;
    if (t < 0) continue;
    const uint64_t row = (uint64_t)(uint32_t)(s.start + (int)i), at = 2 * (head * D + lane * 8);
    const u32x4 k = *reinterpret_cast<const u32x4*>(a.k + row * a.k_stride + at), v = *reinterpret_cast<const u32x4*>(a.v + row * a.v_stride + at);
    const uint32_t page = at_pages.page((uint32_t)t), place = at_pages.place((uint32_t)t);
    const uint64_t word = token_offset(a.cache, page, place) + head * a.cache.head_stride;
    if constexpr (KIND == SPLITZIP_BF16) {
      *reinterpret_cast<u32x4*>(a.cache.k + word + lane * 16) = k;
      *reinterpret_cast<u32x4*>(a.cache.v + word + lane * 16) = v;
    } else {
      uint32_t mk = largest8(k), mv = largest8(v);
#pragma unroll
      for (int o = kLanes / 2; o > 0; o /= 2) {
        mk = max(mk, (uint32_t)__shfl_xor((int)mk, o));
        mv = max(mv, (uint32_t)__shfl_xor((int)mv, o));
      }
      constexpr int kTop = KIND == SPLITZIP_FP8_E5M2 ? kTopE5m2 : kTopE4m3;
      const int bk = scale_byte<kTop>(mk), bv = scale_byte<kTop>(mv);
      *reinterpret_cast<u32x2*>(a.cache.k + word + lane * 8) = to_fp8<KIND>(k, bk);
      *reinterpret_cast<u32x2*>(a.cache.v + word + lane * 8) = to_fp8<KIND>(v, bv);
      if (lane == 0) {
        const uint64_t scale = scale_offset(a.cache, page, place, head);
        a.cache.k_scales[scale] = (uint8_t)bk;
        a.cache.v_scales[scale] = (uint8_t)bv;
      }
    }
  }
}

template <int KIND, int D>
__global__ void __launch_bounds__(kThreads) cache_read_kernel(RowsArgs a) {
  constexpr int kLanes = D / 8, kPairs = kThreads / kLanes;
  const Seq s = seq_at(a.seqs, blockIdx.y);
  const Pages at_pages(a.cache, a.seqs, blockIdx.y);
  const uint32_t lane = threadIdx.x % kLanes, pairs = (uint32_t)s.rows * a.cache.heads;
  for (uint32_t p = blockIdx.x * kPairs + threadIdx.x / kLanes; p < pairs; p += gridDim.x * kPairs) {
    const uint32_t i = p / a.cache.heads, head = p - i * a.cache.heads;
    const int t = s.base + (int)i;
    const uint64_t row = (uint64_t)(uint32_t)(s.start + (int)i), at = 2 * (head * D + lane * 8);
    u32x4 k = {0, 0, 0, 0}, v = {0, 0, 0, 0};   // a row in front of the sequence's first token
    if (t >= 0) {
      const uint32_t page = at_pages.page((uint32_t)t), place = at_pages.place((uint32_t)t);
      const uint64_t word = token_offset(a.cache, page, place) + head * a.cache.head_stride;
      if constexpr (KIND == SPLITZIP_BF16) {
        k = *reinterpret_cast<const u32x4*>(a.cache.k + word + lane * 16);
        v = *reinterpret_cast<const u32x4*>(a.cache.v + word + lane * 16);
      } else {
        const uint64_t scale = scale_offset(a.cache, page, place, head);
        k = from_fp8<KIND>(*reinterpret_cast<const u32x2*>(a.cache.k + word + lane * 8), a.cache.k_scales[scale]);
        v = from_fp8<KIND>(*reinterpret_cast<const u32x2*>(a.cache.v + word + lane * 8), a.cache.v_scales[scale]);
      }
    }
    *reinterpret_cast<u32x4*>(a.k + row * a.k_stride + at) = k;
    *reinterpret_cast<u32x4*>(a.v + row * a.v_stride + at) = v;
  }
}

// The accepted path of a tree of drafted tokens: token base + path[i] becomes token base + i.  A path ascends strictly, so
// path[i] >= i: a token is never written before the ones behind it on the path have been read, as long as every byte of it is
// read and written in the path's order by one thread -- which is what a thread does with its 16 bytes (or its scale) of
// every token.  Entries that do not ascend, or are no rows of the call, end the path.
constexpr uint32_t kMoveMax = 64;   // caches of a launch
struct MoveArgs {
  Cache cache;             // the geometry all of them share
  Seqs seqs;
  const int32_t* path;
  uint32_t path_stride, row_bytes;   // entries per sequence; bytes of a token and head
  struct { uint8_t *k, *v, *k_scales, *v_scales; } at[kMoveMax];
};
__global__ void __launch_bounds__(kThreads) cache_move_kernel(MoveArgs a) {
  const Seq s = seq_at(a.seqs, blockIdx.y);
  const Pages at_pages(a.cache, a.seqs, blockIdx.y);
  const auto& at = a.at[blockIdx.z];
  uint8_t* const words = blockIdx.x ? at.v : at.k;
  uint8_t* const scales = blockIdx.x ? at.v_scales : at.k_scales;
  const uint32_t per_head = a.row_bytes / 16, pieces = per_head * a.cache.heads, of_scales = scales ? a.cache.heads : 0;
  const int32_t* path = a.path + (uint64_t)blockIdx.y * a.path_stride;
  for (uint32_t u = threadIdx.x; u < pieces + of_scales; u += kThreads) {
    const bool is_word = u < pieces;
    const uint32_t head = is_word ? u / per_head : u - pieces, piece = is_word ? u - head * per_head : 0;
    int before = -1;
    for (uint32_t i = 0; i < a.path_stride; ++i) {
      const int from = path[i];
      if (from <= before || from >= s.rows) break;
      before = from;
      const int t = s.base + from, to = s.base + (int)i;
      if (from == (int)i || to < 0) continue;
      const uint32_t p0 = at_pages.page((uint32_t)t), l0 = at_pages.place((uint32_t)t), p1 = at_pages.page((uint32_t)to), l1 = at_pages.place((uint32_t)to);
      if (is_word)
        *reinterpret_cast<u32x4*>(words + token_offset(a.cache, p1, l1) + head * a.cache.head_stride + piece * 16) =
            *reinterpret_cast<const u32x4*>(words + token_offset(a.cache, p0, l0) + head * a.cache.head_stride + piece * 16);
      else
        scales[scale_offset(a.cache, p1, l1, head)] = scales[scale_offset(a.cache, p0, l0, head)];
    }
  }
}

#endif  // SPLITZIP_CACHE_HPP
