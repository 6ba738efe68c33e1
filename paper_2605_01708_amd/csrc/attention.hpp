// SplitZip for MI355X: attention over a paged KV cache.  Part of the single translation unit cache.hip (included inside its
// anonymous namespace, behind cache.hpp).
//
// Row i of a sequence (one token, or one of a tree of drafted tokens, all of them in the cache already) and query head h:
//   x_j = scale q . k_j,  x_j = c tanh(x_j / c) with a cap c,  x_j += slope_h (pos_j - pos_i) with slopes,
//   out = sum_j e^(x_j) v_j / sum_j e^(x_j),  lse = ln sum_j e^(x_j)  over the tokens j that the row may see;
// a row that may see nothing gets zeros and -infinity.
//
// All query heads of a head of the cache, and all rows of a sequence, read the same K and V: they are the rows of one matrix
// product.  A wave takes 16 NT of these rows and 32 tokens at a time, and computes the transposed scores S^T = K Q^T and the
// transposed output O^T = V^T P^T with the 16 x 16 x 32 BF16 matrix instruction.  Transposed, because a lane then holds scores and
// outputs of the one row l % 16 (statistics and rescaling are plain per-lane arithmetic), and because the scores come out of
// the first product in the layout in which the second takes them: lane group g = l / 16 has tokens 4 g .. 4 g + 3 of a
// 16-token tile, and with the tile's row m standing for token 8 (m / 4) + m % 4 of the 32 (and + 4 in the second
// tile) these are tokens 8 g .. 8 g + 7, the lane's eight elements of the second product's K dimension.  No score moves between lanes.
// K is loaded as rows, V as eight tokens times a few elements per lane, transposed in registers by byte permutes.  FP8 words become BF16
// on the way, their scale with them.
//
// The running maximum is one that is at most 2^8 short: it is raised (and what was summed rescaled) only when a score would be
// beyond that, which a wave finds with one comparison and a ballot; weights up to 256 cost nothing in a floating format.  Statistics,
// outputs and the sums over waves and over the parts of a long sequence are held in 32 bits.  V goes into the second product as BF16, and so
// do the weights: up to 16 rows in two parts, which loses nothing that the BF16 result shows (memory's time hides the second product: 64
// sequences of 700 to 8192 tokens 181.1 us, 180.7 with one part; 131072 tokens of E4M3 57.8 and 56.8); of more rows rounded (2^-8 of a weight, as the
// result's own rounding; the error of the result against 64 bits is 0.0021 of it in place of 0.0017), since these kernels are bound by their
// instructions: 16 trees of 64 rows over E5M2 136 us, 161 with two parts, a prompt of 2048 rows 112 and 121.  Their sum is taken before any
// rounding, since lse is a result in 32 bits.
//
// Two kernels: attention_tokens_kernel for up to 16 rows, whose waves take different tokens (memory's speed is all that
// counts), and attention_rows_kernel, whose waves take different rows of the same tokens, staged in LDS.
#ifndef SPLITZIP_ATTENTION_HPP
#define SPLITZIP_ATTENTION_HPP

constexpr uint32_t kStep = 32;          // tokens of a wave at a time
constexpr float kLowest = -3.0e38f;     // the running maximum before the first score (finite: differences stay numbers)
constexpr float kSlack = 8.0f;          // what the running maximum may be short of the largest score, in powers of two
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct AttentionArgs {
  Cache cache;
  Seqs seqs;
  const uint8_t* q;
  uint8_t* out;
  float* lse;                        // [n_rows][q_heads] or null
  uint64_t q_stride, out_stride;     // bytes from row to row
  const float* slopes;               // [q_heads] or null
  const uint64_t* tree;              // [n_rows][tree_words] or null: a chain
  const int32_t* positions;          // [n_rows] or null: base + row
  float* part_out;                   // [workgroup][2][heads_across][kept][D]: parts of sequences that several workgroups share
  float* part_stat;                  // the same, [2] each: maximum (of log2), sum
  float scale, softcap;              // scale >= 0: its sign is in flip_q
  uint32_t flip_q;                   // 0x80008000: the queries change sign
  uint32_t tree_words, window;       // window 0: none
  uint32_t group;                    // query heads per head of the cache
  uint32_t heads_across;             // heads of the cache that a workgroup takes
  uint32_t tile_rows, row_tiles;     // rows of the product that it takes; tiles of them that are dealt out
  uint32_t most_rows, kept;          // rows of a sequence that the launch is cut for, and of a tile that a part is kept of
  uint32_t shares, block_tokens, least_blocks;   // workgroups of the same heads and rows; what is dealt out to them
};

// The arguments once more, where they are needed now and then: read again from where the launch left them, rather than kept in
// scalar registers (or, those used up, in lanes of vector registers) through loops that do not need them.
__device__ inline AttentionArgs args_again() {
  uint64_t at = (uint64_t)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(at));
  AttentionArgs a;
  __builtin_memcpy(&a, (const void*)(const __attribute__((address_space(4))) void*)at, sizeof a);
  return a;
}

__device__ inline int position_of(const AttentionArgs& a, const Seq& s, int i) {
  return a.positions ? a.positions[s.start + i] : s.base + i;
}

// A sequence and the first token that any row of it may see, a multiple of 32: with a window, the one that the row at the lowest
// position sees.  The sequence's blocks count from it.
struct Span : Seq {
  int first;
};
// The lowest position of `rows` rows from `start` on; `each` lanes (a power of two) side by side take them, this one being number `of`.
// Eight at a time: one by one, a call of 16 trees of 64 rows waited 35 us for its positions, one of a prompt of 2048 rows 250.
__device__ inline int lowest(const AttentionArgs& a, int start, int rows, int of, int each) {
  int low = 0x7fffffff;
  for (int i = of; i < rows; i += 8 * each) {
    int at[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) at[k] = a.positions[start + min(i + k * each, rows - 1)];
#pragma unroll
    for (int k = 0; k < 8; ++k) low = min(low, at[k]);
  }
  for (int o = each / 2; o > 0; o /= 2) low = min(low, __shfl_xor(low, o));
  return low;
}
// low: the lowest position of the sequence's rows
__device__ inline int first_from(const AttentionArgs& a, const Seq& s, int low) {
  if (!a.window) return 0;
  const int64_t first = (int64_t)low - (int64_t)a.window + 1;
  const int64_t most = max(min(s.base, s.len), 0);   // drafted tokens lie where their positions say, not where they are stored
  return (int)(max(min(first, most), (int64_t)0) & ~(int64_t)(kStep - 1));
}
// All lanes of a wave together: sequence `seq`, the same for all of them, and sequence at + lane (no rows where there is none).
__device__ inline Span span_at(const AttentionArgs& a, uint32_t lane, uint32_t seq) {
  Span s{seq_at(a.seqs, seq), 0};
  s.first = first_from(a, s, a.window && a.positions ? __builtin_amdgcn_readfirstlane(lowest(a, s.start, s.rows, (int)lane, 64)) : s.base);
  return s;
}
__device__ inline Span spans_at(const AttentionArgs& a, uint32_t lane, uint32_t at) {
  Span s{Seq{0, 0, 0, 0}, 0};
  if (at + lane < a.seqs.n_seqs) static_cast<Seq&>(s) = seq_at(a.seqs, at + lane);
  int low = s.base;
  if (a.window && a.positions) {   // as many lanes for each sequence as there are
    const uint32_t n = min(a.seqs.n_seqs - at, 64u), shift = n > 1 ? (uint32_t)__builtin_clz(n - 1) - 26u : 6u, of = lane >> shift;
    low = lowest(a, __shfl(s.start, (int)of), __shfl(s.rows, (int)of), (int)(lane & ((1u << shift) - 1u)), 1 << shift);
    low = __shfl(low, (int)(lane << shift));
  }
  s.first = first_from(a, s, low);
  return s;
}
// One at least where there are rows: somebody has to write their zeros.
__device__ inline uint32_t blocks_of(const AttentionArgs& a, const Span& s) {
  return s.rows ? max(((uint32_t)(s.len - s.first) + a.block_tokens - 1) / a.block_tokens, 1u) : 0u;
}

// The blocks of all sequences, one sequence behind the other, are dealt out evenly to a.shares workgroups (per heads and tile of
// rows): lengths differ, and a launch that gave every workgroup one part of one sequence would wait for the longest (64 sequences
// of 700 to 8192 tokens: 221 us that way).  Every wave sums the blocks up for itself.
struct Blocks {
  uint32_t shares;     // that get something
  uint32_t each, odd;  // blocks of each, the first `odd` of them one more

  __device__ uint32_t begin(uint32_t share) const { return share * each + min(share, odd); }
  __device__ uint32_t owner(uint32_t block) const {
    const uint32_t longer = odd * (each + 1);
    return block < longer ? block / (each + 1) : odd + (block - longer) / each;
  }
  // mine: sequence `lane`
  __device__ void count(const AttentionArgs& a, uint32_t lane, Span& mine) {
    mine = spans_at(a, lane, 0);
    uint32_t total = wave_last(wave_incl_scan(blocks_of(a, mine)));
    for (uint32_t at = 64; at < a.seqs.n_seqs; at += 64) total += wave_last(wave_incl_scan(blocks_of(a, spans_at(a, lane, at))));
    shares = min(a.shares, (total + a.least_blocks - 1) / a.least_blocks);
    each = total / max(shares, 1u);
    odd = total - each * shares;
  }
  // the sequence that has this block, and the number of its first block
  __device__ void find(const AttentionArgs& a, uint32_t lane, Span mine, uint32_t block, uint32_t& seq, uint32_t& front, Span& s) const {
    uint32_t before = 0;
    for (uint32_t at = 0;; at += 64) {
      if (at) mine = spans_at(a, lane, at);
      const uint32_t n = blocks_of(a, mine), upto = before + wave_incl_scan(n);
      const uint64_t beyond = __ballot(upto > block);
      if (beyond) {
        const int l = __builtin_ctzll(beyond);
        seq = at + (uint32_t)l;
        front = (uint32_t)__builtin_amdgcn_readlane((int)(upto - n), l);
        s = of_lane(mine, l);
        return;
      }
      before = wave_last(upto);
    }
  }
  static __device__ Span of_lane(const Span& s, int l) {
    return Span{Seq{__builtin_amdgcn_readlane(s.start, l), __builtin_amdgcn_readlane(s.rows, l), __builtin_amdgcn_readlane(s.len, l), __builtin_amdgcn_readlane(s.base, l)},
                __builtin_amdgcn_readlane(s.first, l)};
  }
};

// What a workgroup is to do: segment after segment of its blocks, each a piece of one sequence, for heads from `head` on and the rows of
// tile `tile`.
struct Share {
  Span s;
  uint32_t seq, head, tile, rows;   // rows: of the matrix product, the sequence's times the group's query heads
  int begin, end;                   // the segment's tokens
  uint32_t block, blocks, left;     // the segment's first block in the sequence, the sequence's blocks, the workgroup's from here on
  uint32_t slot, wg;                // where the segment's part is kept
  bool whole;                       // the segment is all of the sequence: no part
  int later;                        // segments before this one

  __device__ bool start(uint32_t lane) {
    const AttentionArgs a = args_again();
    // workgroups of the same (share, heads) lie 8 apart, on the same XCD
    wg = blockIdx.x;
    const uint32_t of = wg / 8 / a.row_tiles, groups = a.cache.heads / a.heads_across;
    tile = wg / 8 % a.row_tiles;
    const uint32_t unit = of * 8 + wg % 8, share = unit / groups;
    head = unit % groups * a.heads_across;
    Blocks b;
    Span mine;
    uint32_t front;
    b.count(a, lane, mine);
    if (share >= b.shares) return false;
    const uint32_t from = b.begin(share);
    left = b.begin(share + 1) - from;
    b.find(a, lane, mine, from, seq, front, s);
    later = 0;
    take(a, from - front);
    return true;
  }
  __device__ void take(const AttentionArgs& a, uint32_t at) {
    blocks = blocks_of(a, s);
    rows = (uint32_t)s.rows * a.group;
    block = at;
    if (!blocks) return;
    const uint32_t mine = min(blocks - at, left);
    begin = s.first + (int)(at * a.block_tokens);
    end = at + mine < blocks ? begin + (int)(mine * a.block_tokens) : s.len;
    whole = at == 0 && mine == blocks;
    slot = later ? 1u : 0u;
  }
  // to the next segment
  __device__ bool next(uint32_t lane) {
    const AttentionArgs a = args_again();
    left -= min(blocks - block, left);
    ++later;
    do {
      if (!left) return false;
      seq = (uint32_t)__builtin_amdgcn_readfirstlane((int)(seq + 1));
      s = span_at(a, lane, seq);
      take(a, 0);
    } while (!blocks);
    return true;
  }
  // The segment's first tile of rows, false if there is none, and the next one.  A sequence with more rows than the launch was cut for is taken
  // as a whole by the workgroups that have its first block, every row_tiles-th tile by each: nothing of it needs a place to be kept in.
  __device__ bool first_rows() {
    const AttentionArgs a = args_again();
    tile = wg / 8 % a.row_tiles;
    if (rows > a.most_rows) {
      if (block) return false;
      begin = s.first;
      end = s.len;
      whole = true;
    }
    return (uint64_t)tile * a.tile_rows < rows;
  }
  __device__ bool more_rows() {
    const AttentionArgs a = args_again();
    tile += a.row_tiles;
    return (uint64_t)tile * a.tile_rows < rows;   // (up to most_rows there are no more than row_tiles)
  }
  // The segment's tokens that rows of the tile may see: without a tree, none behind the tile's last row; with a window and no positions, none
  // in front of the first row's, in whole stages of `step` tokens from the segment's begin (so that the last one ends where the segment
  // does).  2048 rows of a prompt under a window of 256: 181 us over all of their tokens, 38 so.
  __device__ void tokens(int& from, int& to, int step) const {
    const AttentionArgs a = args_again();
    from = begin;
    to = end;
    if (!a.tree) to = min(to, s.base + (int)((min((tile + 1) * a.tile_rows, rows) - 1) / a.group) + 1);
    if (a.window && !a.positions) {
      const int64_t lowest = (int64_t)s.base + tile * a.tile_rows / a.group - (int64_t)a.window + 1;
      if (lowest > from) from += (int)(min(lowest, (int64_t)end) - from) & ~(step - 1);
    }
  }
  __device__ uint64_t place(const AttentionArgs& a, uint32_t head_of_group, uint32_t row) const {
    return (((uint64_t)wg * 2 + slot) * a.heads_across + head_of_group) * a.kept + row;
  }
};

// The lane's rows (r0 + 16 n + m of the product) and their operand of the first product.
template <int KIND, int D, int NT>
struct Rows {
  int row[NT];            // row of the sequence (-1: none)
  int low_edge;           // tokens up to here may be out of the window of a row of the workgroup's tile
  bf16x8 q[NT][D / 32];

  __device__ void load(const Share& w, uint32_t r0, uint32_t m, uint32_t g) {
    const AttentionArgs a = args_again();
    low_edge = -1;
    if (a.window) {
      for (uint32_t r = w.tile * a.tile_rows + 16 * g + m; r < min((w.tile + 1) * a.tile_rows, w.rows); r += 64)
        low_edge = max(low_edge, (int)max(min((int64_t)position_of(a, w.s, (int)(r / a.group)) - (int64_t)a.window, (int64_t)w.s.len), (int64_t)-1));
#pragma unroll
      for (int o = 32; o > 0; o /= 2) low_edge = max(low_edge, __shfl_xor(low_edge, o));
    }
    low_edge = __builtin_amdgcn_readfirstlane(low_edge);
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const uint32_t r = r0 + 16 * n + m;
      const bool have = r < w.rows;
      row[n] = have ? (int)(r / a.group) : -1;
      const uint32_t h = w.head * a.group + (have ? r % a.group : 0);
      const uint8_t* at = a.q + (uint64_t)(uint32_t)(w.s.start + max(row[n], 0)) * a.q_stride + 2 * (uint64_t)h * D;
#pragma unroll
      for (int t = 0; t < D / 32; ++t) {
        // FP8 rows are loaded 16 bytes, two steps, at a time: the same order here
        const uint32_t d = KIND == SPLITZIP_BF16 ? 32 * t + 8 * g : 64 * (t / 2) + 16 * g + 8 * (t % 2);
        u32x4 x = {0, 0, 0, 0};
        if (have) x = *reinterpret_cast<const u32x4*>(at + 2 * d) ^ a.flip_q;
        q[n][t] = __builtin_bit_cast(bf16x8, x);
      }
    }
  }
  // whether every row of the tile sees every one of the tokens from t0 on
  __device__ bool see_all(const Share& w, int t0, int tokens) const { return t0 + tokens <= min(w.s.base, w.s.len) && t0 > low_edge; }
  // bit e: row n sees token t8 + e
  __device__ uint32_t seen(const Share& w, int n, int t8) const {
    const AttentionArgs a = args_again();
    if (row[n] < 0) return 0;
    const int behind = min(max(w.s.len - t8, 0), 8), j0 = t8 - w.s.base;   // j0: the row that token t8 is
    uint32_t bits = (1u << behind) - 1u;
    if (j0 > -8) {
      uint32_t b;
      if (a.tree) {
        const uint64_t* words = a.tree + (uint64_t)(uint32_t)(w.s.start + row[n]) * a.tree_words;
        const uint32_t j = (uint32_t)max(j0, 0), at = j / 64, shift = j % 64;
        uint64_t x = at < a.tree_words ? words[at] >> shift : 0;
        if (shift > 56 && at + 1 < a.tree_words) x |= words[at + 1] << (64 - shift);
        b = (uint32_t)x;
      } else {
        b = (1u << min(max(row[n] + 1 - max(j0, 0), 0), 8)) - 1u;
      }
      if (j0 < 0) b = b << -j0 | ((1u << -j0) - 1u);   // tokens in front of the call's own: all rows see them
      bits &= b;
    }
    if (a.window) {
      const int pos = position_of(a, w.s, row[n]);
      if (a.positions && j0 > -8) {
#pragma unroll 1
        for (int e0 = 0; e0 < 8; e0 += 4) {   // four positions at a time (that prompt 163 us, 186 one by one; eight cost all calls registers)
          int at[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) at[e] = a.positions[w.s.start + min(max(j0 + e0 + e, 0), w.s.rows - 1)];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int j = j0 + e0 + e;
            if ((int64_t)pos - (int64_t)(j >= 0 && j < w.s.rows ? at[e] : t8 + e0 + e) >= (int64_t)a.window) bits &= ~(1u << (e0 + e));
          }
        }
      } else {   // tokens lie where they are stored: those of the eight up to pos - window are behind it
        const int64_t behind_it = (int64_t)pos - (int64_t)a.window - (int64_t)t8 + 1;
        bits &= ~0u << (int)min(max(behind_it, (int64_t)0), (int64_t)8);
      }
    }
    return bits;
  }
};

// What the scores of the lane's rows are shaped with.  Loaded once: a load in the loop would wait for all that the loop has asked for ahead.
template <int NT>
struct Bias {
  float slope[NT];   // times log2 e; 0: no bias
  int pos[NT];
  __device__ void load(const Share& w, const int (&row)[NT], uint32_t r0, uint32_t m) {
    const AttentionArgs a = args_again();
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const bool have = a.slopes && row[n] >= 0;
      slope[n] = have ? a.slopes[w.head * a.group + (r0 + 16 * n + m) % a.group] * kLog2e : 0.0f;
      pos[n] = have ? position_of(a, w.s, row[n]) : 0;
    }
  }
};

constexpr float kSmallCap = 128.0f;
// the scores' way into the exponent of two
__device__ inline float shaped(const AttentionArgs& a, float x, float slope_log2, float far) {
  x *= a.scale;
  if (a.softcap > 0.0f) {
    // tanh(y) = 1 - 2 / (1 + e^2y): its absolute error of 1e-7 times the cap is one of the exponent
    const float e = __builtin_amdgcn_exp2f(x * (2.0f * kLog2e / a.softcap));
    const float capped = a.softcap - (2.0f * a.softcap) * __builtin_amdgcn_rcpf(1.0f + e);
    if (__builtin_expect(a.softcap > kSmallCap, 0)) {   // ... which wide caps make large: there, the series where y is below a quarter
      const float y = x * __builtin_amdgcn_rcpf(a.softcap), t = y * y;
      x = t < 0.0625f ? x * (1.0f - t * (1.0f / 3.0f - t * (2.0f / 15.0f - t * (17.0f / 315.0f)))) : capped;
    } else {
      x = capped;
    }
  }
  return x * kLog2e - slope_log2 * far;
}

// the larger of two, the other one of a NaN: one instruction, where fmaxf is two, since it makes its operands' NaN quiet
__device__ inline float larger(float x, float y) { return __builtin_amdgcn_fmed3f(x, y, __builtin_inff()); }

__device__ inline f32x4 mfma(const bf16x8& x, const bf16x8& y, const f32x4& c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, y, c, 0, 0, 0); }
__device__ inline bf16x8 as_bf16(const u32x4& x) { return __builtin_bit_cast(bf16x8, x); }

// bytes of a pair of tokens' elements 2 i, 2 i + 1 (BF16) into the pair of element 2 i and that of 2 i + 1
__device__ inline uint32_t evens(uint32_t t0, uint32_t t1) { return byte_perm(t1, t0, 0x05040100u); }
__device__ inline uint32_t odds(uint32_t t0, uint32_t t1) { return byte_perm(t1, t0, 0x07060302u); }

// Nothing is fetched ahead across this: on the ways that are rarely taken, registers count, which the usual way needs.
__device__ inline void one_at_a_time() { asm volatile("" ::: "memory"); }

// What a wave has of its rows: outputs (tile j of D / 16: an element per lane and register), the sum of the weights of the lane's own
// tokens and the running maximum, of powers of two.
template <int D, int NT>
struct State {
  f32x4 acc[NT][D / 16];
  float sum[NT], top[NT];
  __device__ void clear() {
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      top[n] = kLowest;
      sum[n] = 0.0f;
#pragma unroll
      for (int j = 0; j < D / 16; ++j) acc[n][j] = f32x4{0, 0, 0, 0};
    }
  }

  // Scores x of the 32 tokens from t0 on (the lane's eight from t0 + 8 g on), as they come out of the product:
  // capped and biased, in powers of two
  static __device__ void shape(const Share& w, const Bias<NT>& bias, f32x4 (&x)[NT][2], int t8) {
    const AttentionArgs a = args_again();
    int at[8];   // positions of the lane's tokens
    if (a.slopes) {
#pragma unroll
      for (int e = 0; e < 8; ++e) at[e] = t8 + e;
      if (__builtin_expect(__ballot(t8 + 7 >= w.s.base) != 0, 0)) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int j = t8 + e - w.s.base;
          if (j >= 0 && t8 + e < w.s.len) at[e] = position_of(a, w.s, j);
        }
      }
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll   // (2^30 and -2^30 are 2^31 apart, one more than an integer holds; the one below becomes 2^31 as a float)
      for (int e = 0; e < 8; ++e) x[n][e / 4][e % 4] = shaped(a, x[n][e / 4][e % 4], bias.slope[n], a.slopes ? (float)__builtin_elementwise_sub_sat(bias.pos[n], at[e]) : 0.0f);
    }
  }
  // without the tokens that a row does not see
  template <int KIND>
  static __device__ void mask(const Share& w, const Rows<KIND, D, NT>& r, f32x4 (&x)[NT][2], int t8) {
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const uint32_t seen = r.seen(w, n, t8);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[n][e / 4][e % 4] = seen >> e & 1 ? x[n][e / 4][e % 4] : -__builtin_inff();
    }
  }
  static __device__ float highest(const f32x4 (&x)[2]) {
    return larger(larger(larger(x[0][0], x[0][1]), larger(x[0][2], x[0][3])), larger(larger(x[1][0], x[1][1]), larger(x[1][2], x[1][3])));
  }
  // The running maximum, raised if need be; high: the lane's highest score of the tokens to come, in powers of two.
  __device__ void raise(const float (&high)[NT]) {
    bool need = false;
#pragma unroll
    for (int n = 0; n < NT; ++n) need |= high[n] > top[n] + kSlack;
    if (__builtin_expect(__ballot(need) != 0, 0)) {
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        float h = high[n];
        h = fmaxf(h, __shfl_xor(h, 16));
        h = fmaxf(h, __shfl_xor(h, 32));
        const float now = fmaxf(top[n], h), less = __builtin_amdgcn_exp2f(top[n] - now);
        top[n] = now;
        sum[n] *= less;
#pragma unroll
        for (int j = 0; j < D / 16; ++j) acc[n][j] *= less;
      }
    }
  }
  // The weights of the lane's eight tokens and their sum; powers of two are the scores times c.  N = 1: weights rounded to BF16.  N = 2: each
  // in two parts of BF16, 2^-15 of it short at most; the first is cut from a little less than the weight, so that both are above 0
  // where the weight is, and an infinity of V stays one in either product.
  template <int N>
  __device__ void weigh(float c, const f32x4 (&x)[NT][2], bf16x8 (&p)[N][NT]) {
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      float e[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) e[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[n][i / 4][i % 4], c, -top[n]));
      sum[n] += ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));
      if constexpr (N == 2) {
        uint32_t first[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          first[i] = __float_as_uint(e[i] * (1.0f - 0x1p-9f));
          e[i] -= __uint_as_float(first[i] & 0xffff0000u);
        }
        p[1][n] = as_bf16(u32x4{odds(first[0], first[1]), odds(first[2], first[3]), odds(first[4], first[5]), odds(first[6], first[7])});
      }
      p[0][n] = as_bf16(u32x4{bf16_pair(e[0], e[1]), bf16_pair(e[2], e[3]), bf16_pair(e[4], e[5]), bf16_pair(e[6], e[7])});
    }
  }

  __device__ float total(int n) const {   // of all the wave's tokens
    const float x = sum[n] + __shfl_xor(sum[n], 16);
    return x + __shfl_xor(x, 32);
  }
  template <int N>
  __device__ void add(int j, const bf16x8& v, const bf16x8 (&p)[N][NT]) {
#pragma unroll
    for (int k = 0; k < N; ++k)
#pragma unroll
      for (int n = 0; n < NT; ++n) acc[n][j] = mfma(v, p[k][n], acc[n][j]);
  }
  // A token that some row does not see may hold anything, and 0 times an infinity or a NaN is no 0: where there are such tokens, V goes
  // into the product without these words (finite_only), and what rows do see of them is added here, from memory, when the
  // tokens from `begin` to `end` are done, which went in `step` at a time.  (A weight that is not 0 does not change what is added.)  element(j, i): which element the lane has in acc[n][j][i].
  template <int KIND, typename E>
  __device__ void add_odd(const Share& w, const Rows<KIND, D, NT>& r, int begin, int end, int step, const E& element) {
    const AttentionArgs a = args_again();
    const Pages pages(a.cache, a.seqs, w.seq);
#pragma unroll 1
    for (int t0 = begin; t0 < end; t0 += step) {
      if (r.see_all(w, t0, step)) continue;
#pragma unroll 1
      for (int t = t0; t < min(t0 + step, min(end, w.s.len)); ++t) {
        const uint32_t page = pages.page((uint32_t)t), place = pages.place((uint32_t)t);
        const uint8_t* at = a.cache.v + token_offset(a.cache, page, place) + w.head * a.cache.head_stride;
        uint32_t byte = 0;
        if constexpr (KIND != SPLITZIP_BF16) byte = a.cache.v_scales[scale_offset(a.cache, page, place, w.head)];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          const bool mine = r.seen(w, n, t & ~7) >> (t & 7) & 1;
#pragma unroll
          for (int j = 0; j < D / 16; ++j) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              uint32_t v;
              if constexpr (KIND == SPLITZIP_BF16) v = reinterpret_cast<const uint16_t*>(at)[element(j, i)];
              else v = fp8_pair_to_bf16<KIND, false>(at[element(j, i)], byte) & 0xffffu;
              acc[n][j][i] += mine && (v & 0x7f80u) == 0x7f80u ? __uint_as_float(v << 16) : 0.0f;
            }
            one_at_a_time();
          }
        }
      }
    }
  }
};

// halves of a pair of tokens that are among the sequence's
__device__ inline uint32_t inside(int t, int len) { return (t < len ? 0xffffu : 0u) | (t + 1 < len ? 0xffff0000u : 0u); }
// zeros for the infinities and NaN of N registers of V (element j of the eight tokens from t8 on in vt[j]); whether a token of the sequence had one
template <int N>
__device__ inline bool finite_only(u32x4 (&vt)[N], int t8, int len) {
  uint32_t any = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t in = inside(t8 + 2 * i, len);
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const uint32_t odd = ((vt[j][i] & 0x7f807f80u) + 0x00800080u) & 0x80008000u;   // an exponent of ones carries into the sign's place
      vt[j][i] &= ~(odd - (odd >> 15) | odd);
      any |= odd & in;
    }
  }
  return any != 0;
}

__device__ inline float lse_of(float top, float total) { return total != 0.0f ? (top + __builtin_amdgcn_logf(total)) * kLn2 : -__builtin_inff(); }
__device__ inline float one_over(float total) { return total != 0.0f ? 1.0f / total : 0.0f; }   // (a NaN is no 0)

// Up to 16 rows: memory's speed is all that counts.  A wave belongs to one head of the cache; the four of a workgroup take two heads (or, of an
// odd number of heads, one) and every second (or fourth) stage of tokens, so that heads of a token, which lie side by
// side, are read at the same time.  K and V go from memory straight into a piece of LDS of the wave's own, in whole rows (a load of the
// matrix operand itself would take 16 bytes from each of 16 rows at a time), from there into registers, and while the wave
// works on those the next tokens are on their way to the same place: no barrier, 128 KB of a CU's LDS in flight.
//
// Bound by memory where there is enough to read: 64 sequences of 700 to 8192 tokens, 8 heads of 128 in BF16, 1.17 GB in 180 us (6.5 TB/s; reading
// alone reaches 7.1).  Short of that by what a launch has before its first and behind its last load (the tables' and lengths' way to the first
// address 5 us, the join 5 to 7): 131072 tokens of E4M3, 270 MB, in 51 and 6 us.
template <int KIND, int D>
struct Stream {
  // A stage is 16 KB per wave, two workgroups per CU (32 tokens of 256 BF16 elements: 32 KB, one).
  static constexpr int ES = KIND == SPLITZIP_BF16 ? 2 : 1;
  static constexpr int kRow = D * ES;                                    // bytes of a token
  static constexpr int kTokens = 16384 / (2 * kRow) < 32 ? 32 : 16384 / (2 * kRow);   // of a stage
  static constexpr int kHalf = kTokens * kRow;                           // bytes of K, or V, of a stage
  static constexpr int kSteps = kTokens / (int)kStep;
  static constexpr int kUnits = kRow / 16;                               // 16-byte units of a row
  static constexpr int KS = D / 32, DV = D / 16;
  static constexpr int KW = KS * ES / 2;                                 // units of a row of K per lane
  static constexpr int VB = DV * ES;                                     // bytes of a token of V per lane
  static constexpr int VW = VB / 4;

  // Rows of K lie in the order of the tokens, their units permuted so that the 16 rows of an operand (of the tile's row m: token
  // 8 (m / 4) + m % 4, the other tile's 4 further) lie in 16 different units of the banks.
  __device__ static uint32_t k_key(uint32_t token) {
    const uint32_t mi = token / 8 % 4 * 4 + token % 4;
    return kUnits >= 16 ? mi : mi / (16 / kUnits);
  }
  // Rows of V: those of the second and fourth eight in pairs the other way round where four of them (one of each eight) are read at a time
  // and a row is half of the banks.
  __device__ static uint32_t v_row(uint32_t token) { return kUnits == 8 ? token ^ (token / 8 & 1) : token; }

  // asks for the stage from token t0 on; pages: lane l has the page of its 8 l-th token
  __device__ static void ask(const Cache& c, const Pages& at_pages, const uint8_t* k_base, const uint8_t* v_base, uint32_t pages, int t0,
                             uint32_t last8, uint8_t* lds, uint32_t lane) {
#pragma unroll
    for (int i = 0; i < kHalf / 1024; ++i) {
      const uint32_t unit = (uint32_t)i * 64 + lane, row = unit / kUnits, at = unit % kUnits;   // where this lane's 16 bytes come to lie
      // (rows of 128 bytes or more: the eight tokens are the same ones for all lanes)
      const uint32_t eight = kUnits >= 8 ? (uint32_t)i * 64 / kUnits / 8 : row / 8;
      uint32_t page;
      if constexpr (kUnits >= 8) page = (uint32_t)__builtin_amdgcn_readlane((int)pages, i * 64 / kUnits / 8);
      else page = (uint32_t)__shfl((int)pages, (int)(row / 8));
      const uint64_t from = token_offset(c, page, at_pages.place(min((uint32_t)t0 + 8 * eight, last8)));
      const uint32_t k_off = row % 8 * c.token_stride + (at ^ k_key(row)) * 16;
      const uint32_t v_off = v_row(row) % 8 * c.token_stride + at * 16;
      load_to_lds(k_base + from + k_off, lds + i * 1024);
      load_to_lds(v_base + from + v_off, lds + kHalf + i * 1024);
    }
  }
};

template <int KIND, int D, bool PLAIN>
__global__ void __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(Stream<KIND, D>::kHalf > 8192 ? 1 : 2))) attention_tokens_kernel(AttentionArgs args) {
  using S = Stream<KIND, D>;
  constexpr int ES = S::ES, KS = S::KS, DV = S::DV, KW = S::KW, VW = S::VW;
  __shared__ __attribute__((aligned(1024))) uint8_t lds_all[kWaves][2 * S::kHalf];
  __shared__ float lds_stat[kWaves][16][2];
  const uint32_t lane = threadIdx.x % 64, wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / 64)), m = lane % 16, g = lane / 16;
  Share w;
  if (!w.start(lane)) return;
  const Cache c = args.cache;
  const float scale = PLAIN ? args.scale * kLog2e : 1.0f;   // PLAIN: scores without cap and bias, their powers of two the products times this
  const uint32_t hw = args.heads_across, tw = kWaves / hw, turn = wave / hw;   // heads of the workgroup, waves of a head, which of them
  w.head += wave % hw;
  const uint8_t *k_base = c.k + w.head * c.head_stride, *v_base = c.v + w.head * c.head_stride;
  uint8_t* const mine = lds_all[wave];
  const int stride = (int)tw * S::kTokens;

  do {
    if (!w.first_rows()) continue;
    do {
      const uint32_t last8 = (uint32_t)(w.s.len - 1) & ~7u;   // tokens behind the sequence's end are read at its last eight
      const Pages at_pages(c, args.seqs, w.seq);
      const auto ask_pages = [&](int t0) { return at_pages.entry(min((uint32_t)t0 + 8 * (lane % (S::kTokens / 8)), last8)); };
      u32x2 k_scales[S::kSteps], v_scales[S::kSteps];
      const auto ask_scales = [&](uint32_t pages, int t0) {
        if constexpr (ES == 1) {
  #pragma unroll
          for (int u = 0; u < S::kSteps; ++u) {
            const uint32_t k4 = 4 * u + m / 4, v4 = 4 * u + g;
            const uint32_t k_place = at_pages.place(min((uint32_t)t0 + 8 * k4, last8)), v_place = at_pages.place(min((uint32_t)t0 + 8 * v4, last8));
            k_scales[u] = *reinterpret_cast<const u32x2*>(c.k_scales + scale_offset(c, (uint32_t)__shfl((int)pages, (int)k4), k_place, w.head));
            v_scales[u] = *reinterpret_cast<const u32x2*>(c.v_scales + scale_offset(c, (uint32_t)__shfl((int)pages, (int)v4), v_place, w.head));
          }
        }
      };
      int t0 = w.begin + (int)turn * S::kTokens;
      uint32_t pages = 0;
      if (t0 < w.end) {
        pages = ask_pages(t0);
        pages = at_pages.clamped(pages);
        S::ask(c, at_pages, k_base, v_base, pages, t0, last8, mine, lane);
        ask_scales(pages, t0);
        if (t0 + stride < w.end) pages = ask_pages(t0 + stride);
      }
      Rows<KIND, D, 1> r;
      r.load(w, w.tile * 16, m, g);
      Bias<1> bias;
      if constexpr (!PLAIN) bias.load(w, r.row, w.tile * 16, m);
      State<D, 1> st;
      st.clear();
      bool odd = false;   // words of V were left out
  #pragma unroll 1
      for (; t0 < w.end; t0 += stride) {
        memory_arrived();
        u32x4 k[S::kSteps][2][KW];
        uint32_t v[S::kSteps][8][VW];
  #pragma unroll
        for (int u = 0; u < S::kSteps; ++u) {
  #pragma unroll
          for (int b = 0; b < 2; ++b)
  #pragma unroll
            for (int i = 0; i < KW; ++i) {
              const uint32_t token = 32 * u + 8 * (m / 4) + 4 * b + m % 4;
              k[u][b][i] = *reinterpret_cast<const u32x4*>(mine + token * S::kRow + ((4 * i + g) ^ S::k_key(token)) * 16);
            }
  #pragma unroll
          for (int e = 0; e < 8; ++e)
            __builtin_memcpy(v[u][e], __builtin_assume_aligned(mine + S::kHalf + S::v_row(32 * u + 8 * g + e) * S::kRow + S::VB * m, S::VB < 16 ? S::VB : 16), S::VB);
        }
        u32x2 ks[S::kSteps], vs[S::kSteps];
  #pragma unroll
        for (int u = 0; u < S::kSteps; ++u) {
          ks[u] = k_scales[u];
          vs[u] = v_scales[u];
        }
        lds_read();   // into registers: the place is free
        if (t0 + stride < w.end) {
          pages = at_pages.clamped(pages);
          S::ask(c, at_pages, k_base, v_base, pages, t0 + stride, last8, mine, lane);
          ask_scales(pages, t0 + stride);
          if (t0 + 2 * stride < w.end) pages = ask_pages(t0 + 2 * stride);
        }
  #pragma unroll
        for (int u = 0; u < S::kSteps; ++u) {
          const int tu = t0 + u * (int)kStep;
          if (tu >= w.end) break;
          f32x4 x[1][2];
  #pragma unroll
          for (int b = 0; b < 2; ++b) {
            x[0][b] = f32x4{0, 0, 0, 0};
  #pragma unroll
            for (int t = 0; t < KS; ++t) {
              if constexpr (ES == 2) {
                x[0][b] = mfma(as_bf16(k[u][b][t]), r.q[0][t], x[0][b]);
              } else {
                const u32x2 words = {k[u][b][t / 2][t % 2 * 2], k[u][b][t / 2][t % 2 * 2 + 1]};
                x[0][b] = mfma(as_bf16(from_fp8<KIND>(words, ks[u][b] >> (8 * (m % 4)) & 0xffu)), r.q[0][t], x[0][b]);
              }
            }
          }
          const bool all = r.see_all(w, tu, (int)kStep);
          const int t8 = tu + (int)(8 * g);
          if constexpr (!PLAIN) st.shape(w, bias, x, t8);
          if (__builtin_expect(!all, 0)) st.mask(w, r, x, t8);
          st.raise({st.highest(x[0]) * scale});
          bf16x8 p[2][1];
          st.weigh(scale, x, p);
          u32x4 vt[DV];   // element j of the eight tokens
  #pragma unroll
          for (int i = 0; i < 4; ++i) {
  #pragma unroll
            for (int j = 0; j < DV; j += 2) {
              uint32_t w0, w1;
              if constexpr (ES == 2) {
                w0 = v[u][2 * i][j / 2];
                w1 = v[u][2 * i + 1][j / 2];
              } else {
                const uint32_t b0 = vs[u][i / 2] >> (16 * (i % 2)) & 0xffu, b1 = vs[u][i / 2] >> (16 * (i % 2) + 8) & 0xffu;
                w0 = j % 4 ? fp8_pair_to_bf16<KIND, true>(v[u][2 * i][j / 4], b0) : fp8_pair_to_bf16<KIND, false>(v[u][2 * i][j / 4], b0);
                w1 = j % 4 ? fp8_pair_to_bf16<KIND, true>(v[u][2 * i + 1][j / 4], b1) : fp8_pair_to_bf16<KIND, false>(v[u][2 * i + 1][j / 4], b1);
              }
              vt[j][i] = evens(w0, w1);
              vt[j + 1][i] = odds(w0, w1);
            }
          }
          if (__builtin_expect(!all, 0)) odd |= finite_only(vt, t8, w.s.len);
  #pragma unroll
          for (int j = 0; j < DV; ++j) st.add(j, as_bf16(vt[j]), p);
        }
      }
      if (__builtin_expect(__ballot(odd) != 0, 0)) {
        const auto element = [&](int j, int i) { return DV * (4 * g + i) + j; };
        for (int t = w.begin + (int)turn * S::kTokens; t < w.end; t += stride) st.add_odd(w, r, t, min(t + S::kTokens, w.end), (int)kStep, element);
      }

      // the waves of a head (two or four) together; lane (m, g) has elements DV (4 g + i) + j of row m in acc[j][i]
      float total = st.total(0);
      if (g == 0) {
        lds_stat[wave][m][0] = st.top[0];
        lds_stat[wave][m][1] = total;
      }
      f32x4* out = reinterpret_cast<f32x4*>(mine) + lane;
  #pragma unroll
      for (int j = 0; j < DV; ++j) out[64 * j] = st.acc[0][j];
      lds_barrier();
      if (turn == 0) {
        float high = st.top[0];
        for (uint32_t v = 1; v < tw; ++v) high = fmaxf(high, lds_stat[wave + v * hw][m][0]);
        const float f0 = __builtin_amdgcn_exp2f(st.top[0] - high);
        st.top[0] = high;
        total *= f0;
  #pragma unroll
        for (int j = 0; j < DV; ++j) st.acc[0][j] *= f0;
        for (uint32_t v = 1; v < tw; ++v) {
          const float f = __builtin_amdgcn_exp2f(lds_stat[wave + v * hw][m][0] - high);
          total += f * lds_stat[wave + v * hw][m][1];
          const f32x4* from = reinterpret_cast<const f32x4*>(lds_all[wave + v * hw]) + lane;
  #pragma unroll
          for (int j = 0; j < DV; ++j) st.acc[0][j] += f * from[64 * j];
        }
      }
      lds_barrier();   // (the next tile of rows writes there)
      const uint32_t at = w.tile * 16 + m;
      if (turn == 0 && at < w.rows) {
        const AttentionArgs a = args_again();
        const uint32_t q_heads = a.cache.heads * a.group, h = w.head * a.group + at % a.group;
        const uint64_t out_row = (uint64_t)(uint32_t)(w.s.start + (int)(at / a.group));
        if (w.whole) {
          const float f = one_over(total);
          uint8_t* to = a.out + out_row * a.out_stride + 2 * ((uint64_t)h * D + 4 * DV * g);
  #pragma unroll
          for (int i = 0; i < 4; ++i)
  #pragma unroll
            for (int j = 0; j < DV; j += 4)
              *reinterpret_cast<u32x2*>(to + 2 * (DV * i + j)) = u32x2{bf16_pair(st.acc[0][j][i] * f, st.acc[0][j + 1][i] * f), bf16_pair(st.acc[0][j + 2][i] * f, st.acc[0][j + 3][i] * f)};
          if (g == 0 && a.lse) a.lse[out_row * q_heads + h] = lse_of(st.top[0], total);
        } else {
          const uint64_t place = w.place(a, wave % hw, m);
          float* to = a.part_out + place * D + 4 * DV * g;
  #pragma unroll
          for (int i = 0; i < 4; ++i)
  #pragma unroll
            for (int j = 0; j < DV; j += 4)
              *reinterpret_cast<f32x4*>(to + DV * i + j) = f32x4{st.acc[0][j][i], st.acc[0][j + 1][i], st.acc[0][j + 2][i], st.acc[0][j + 3][i]};
          if (g == 0) {
            a.part_stat[2 * place] = st.top[0];
            a.part_stat[2 * place + 1] = total;
          }
        }
      }
    } while (w.more_rows());
  } while (w.next(lane));
}

// More rows: the W waves of a workgroup take 16 NT rows each of the same tokens.  Those are staged in LDS, 4 KB per wave at a time, as the
// operands of the matrix instruction that they are (lane after lane, 16 bytes each: written and read without a bank
// conflict), FP8 words converted and V transposed once for all waves.  Half of the waves stage four operands of K each, the others
// four of V; a wave asks for its piece of the next stage before it works on this one, which is written in the other half of LDS: one
// barrier a stage, since who writes a half has passed the barrier behind which nobody reads it.
//
// Bound by the matrix instructions' rate with what surrounds them, hardly ever by memory: 16 sequences of 3001 to 8192 E5M2 tokens under 256 rows (64 drafts of four
// query heads) of 8 heads of 128, 94 GFLOP, in 134 us (0.7 PFLOP/s; a large library product of BF16 reaches 1.2), of which, measured apart, the products and
// exponentials are 86, loads and their conversion 14, and prologue, parts and waiting the rest; joining takes 16 more.
template <int KIND, int D, int W>
struct Stage {
  static constexpr int ES = KIND == SPLITZIP_BF16 ? 2 : 1;
  static constexpr int KS = D / 32, DV = D / 16;
  static constexpr int kTokens = W * 1024 / D, kUnits = kTokens / (int)kStep;
  static constexpr int kV = 2 * W;   // operands of K, and of V behind them
  static_assert(kTokens >= (int)kStep, "a stage has 32 tokens at least");
  uint32_t w[8 * ES];   // K: 16-byte runs of rows, operands 4 s .. 4 s + 3 (two of them in 16 bytes of FP8); V: four elements of eight tokens
  u32x2 scales;

  // piece s of K: operand f = 4 s + i is step f % KS of the tile f / KS of 16 tokens
  __device__ static uint32_t k_group(uint32_t s, uint32_t m) { return 4 * s / KS / 2 * 32 + 8 * (m / 4); }
  // (base: of the head, the lane's token of eight and its 16 bytes)
  __device__ void load_k(const Cache& c, const uint8_t* base, uint32_t page, uint32_t place, uint32_t head, uint32_t s) {
    const uint8_t* at = base + token_offset(c, page, place);
#pragma unroll
    for (int i = 0; i < 2 * ES; ++i) {
      const uint32_t f = 4 * s + (ES == 2 ? i : 2 * i);
      const u32x4 x = *reinterpret_cast<const u32x4*>(at + (uint64_t)(f / KS % 2 * 4) * c.token_stride + (ES == 2 ? f % KS : f % KS / 2) * 64);
#pragma unroll
      for (int j = 0; j < 4; ++j) w[4 * i + j] = x[j];
    }
    if constexpr (ES == 1) scales = *reinterpret_cast<const u32x2*>(c.k_scales + scale_offset(c, page, place, head));
  }
  __device__ void store_k(u32x4* to, uint32_t s, uint32_t m) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (ES == 2) {
        to[64 * i] = u32x4{w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]};
      } else {
        const uint32_t pair = (4 * s + i) / KS % 2 ? scales[1] : scales[0];
        to[64 * i] = from_fp8<KIND>(u32x2{w[2 * i], w[2 * i + 1]}, pair >> (8 * (m % 4)) & 0xffu);
      }
    }
  }
  // piece s of V: 64 elements (block s % (D / 64)) of 32 tokens; a lane has elements 4 m .. 4 m + 3 of them of tokens 8 g ..
  __device__ static uint32_t v_group(uint32_t s, uint32_t g) { return s / (D / 64) * 32 + 8 * g; }
  __device__ void load_v(const Cache& c, const uint8_t* base, uint32_t page, uint32_t place, uint32_t head) {
    const uint8_t* at = base + token_offset(c, page, place);
#pragma unroll
    for (int e = 0; e < 8; ++e) __builtin_memcpy(w + ES * e, __builtin_assume_aligned(at + (uint64_t)e * c.token_stride, 4 * ES), 4 * ES);
    if constexpr (ES == 1) scales = *reinterpret_cast<const u32x2*>(c.v_scales + scale_offset(c, page, place, head));
  }
  // guarded: without infinities and NaN; true if there were some
  __device__ bool store_v(u32x4* to, bool guarded, int t8, int len) const {
    u32x4 vt[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t x0[2], x1[2];
      if constexpr (ES == 2) {
        x0[0] = w[4 * i];
        x0[1] = w[4 * i + 1];
        x1[0] = w[4 * i + 2];
        x1[1] = w[4 * i + 3];
      } else {
        const uint32_t b0 = scales[i / 2] >> (16 * (i % 2)) & 0xffu, b1 = scales[i / 2] >> (16 * (i % 2) + 8) & 0xffu;
        x0[0] = fp8_pair_to_bf16<KIND, false>(w[2 * i], b0);
        x0[1] = fp8_pair_to_bf16<KIND, true>(w[2 * i], b0);
        x1[0] = fp8_pair_to_bf16<KIND, false>(w[2 * i + 1], b1);
        x1[1] = fp8_pair_to_bf16<KIND, true>(w[2 * i + 1], b1);
      }
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        vt[2 * j][i] = evens(x0[j], x1[j]);
        vt[2 * j + 1][i] = odds(x0[j], x1[j]);
      }
    }
    bool odd = false;
    if (__builtin_expect(guarded, 0)) odd = finite_only(vt, t8, len);
#pragma unroll
    for (int j = 0; j < 4; ++j) to[64 * j] = vt[j];
    return odd;
  }
};

template <int KIND, int D, int W, int NT, bool PLAIN>
__global__ void __launch_bounds__(64 * W) __attribute__((amdgpu_waves_per_eu(W == 4 ? 3 : 2))) attention_rows_kernel(AttentionArgs args) {
  using S = Stage<KIND, D, W>;
  constexpr int KS = S::KS, DV = S::DV, kTokens = S::kTokens, kUnits = S::kUnits;
  __shared__ u32x4 lds[2][W * 4 * 64];
  // The workgroup's last tile of rows (of the even ones, and of the odd ones) in whose stages words of V were left out.  They are counted from 1:
  // what a tile finds here is its own, since a place is written again by the second tile after it, two barriers on.
  __shared__ uint32_t lds_odd[2];
  const uint32_t lane = threadIdx.x % 64, wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / 64)), m = lane % 16, g = lane / 16;
  Share w;
  if (!w.start(lane)) return;
  const Cache c = args.cache;
  const float scale = PLAIN ? args.scale * kLog2e : 1.0f;
  // Of the two waves that a SIMD has of the workgroup one goes first, or both would be at the same instructions after every barrier: the
  // matrix ones, then the others (64 drafts over BF16: 159 us without, 150 with).
  if (W == 8 && wave >= 4) __builtin_amdgcn_s_setprio(1);
  const bool of_k = wave < W / 2;
  const uint32_t piece = wave % (W / 2);
  const uint8_t* const base = of_k ? c.k + w.head * c.head_stride + (uint64_t)(m % 4) * c.token_stride + 16 * g
                                   : c.v + w.head * c.head_stride + S::ES * (64 * (piece % (D / 64)) + 4 * m);
  const uint32_t group = of_k ? S::k_group(piece, m) : S::v_group(piece, g);   // the lane's eight tokens of a stage
  if (threadIdx.x < 2) lds_odd[threadIdx.x] = 0;
  lds_barrier();
  uint32_t turn = 0;

  do {
    if (!w.first_rows()) continue;
    do {
      ++turn;
      int from, to;
      w.tokens(from, to, kTokens);
      const uint32_t last8 = (uint32_t)(w.s.len - 1) & ~7u;   // tokens behind the sequence's end are read at its last eight
      const Pages at_pages(c, args.seqs, w.seq);
      const uint32_t r0 = (w.tile * W + wave) * 16 * NT;
      const bool active = r0 < w.rows;
      Rows<KIND, D, NT> r;
      State<D, NT> st;
      S stage;
      uint32_t page = 0;
      const auto ask_page = [&](int t0) {
        if (t0 < to) page = at_pages.entry(min((uint32_t)t0 + group, last8));
      };
      const auto ask = [&](int t0) {
        if (t0 >= to) return;
        const uint32_t place = at_pages.place(min((uint32_t)t0 + group, last8));
        const uint32_t in_pool = at_pages.clamped(page);
        if (of_k) stage.load_k(c, base, in_pool, place, w.head, piece);
        else stage.load_v(c, base, in_pool, place, w.head);
      };
      const auto store = [&](int t0, int buf) {
        if (t0 >= to) return;
        u32x4* to = lds[buf] + 64 * (of_k ? 4 * piece : S::kV + 4 * piece) + lane;
        if (of_k) stage.store_k(to, piece, m);
        else if (__builtin_expect(stage.store_v(to, !r.see_all(w, t0, kTokens), t0 + (int)group, w.s.len), 0)) lds_odd[turn % 2] = turn;
      };
      // the scores of 32 tokens, unit u of a stage
      const auto scores = [&](f32x4 (&x)[NT][2], const u32x4* at) {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
#pragma unroll
          for (int n = 0; n < NT; ++n) x[n][b] = f32x4{0, 0, 0, 0};
#pragma unroll
          for (int t = 0; t < KS; ++t) {
            const bf16x8 k = as_bf16(at[64 * (b * KS + t)]);
#pragma unroll
            for (int n = 0; n < NT; ++n) x[n][b] = mfma(k, r.q[n][t], x[n][b]);
          }
        }
      };
      ask_page(from);
      ask(from);
      ask_page(from + kTokens);
      r.load(w, r0, m, g);
      Bias<NT> bias;
      if constexpr (!PLAIN) bias.load(w, r.row, r0, m);
      st.clear();
      int buf = 0;
#pragma unroll 1
      for (int t0 = from; t0 < to; t0 += kTokens, buf ^= 1) {
        store(t0, buf);
        ask(t0 + kTokens);
        ask_page(t0 + 2 * kTokens);
        lds_barrier();
        if (!active) continue;
        const u32x4* const at = lds[buf] + lane;
        // all units of the stage at a time, so that there is one question about the maximum, and enough to do between its answers
        const bool all = r.see_all(w, t0, kTokens);
        f32x4 x[kUnits][NT][2];
        float high[NT];
#pragma unroll
        for (int u = 0; u < kUnits; ++u) {
          const int t8 = t0 + u * (int)kStep + (int)(8 * g);
          scores(x[u], at + 64 * 2 * KS * u);
          if constexpr (!PLAIN) st.shape(w, bias, x[u], t8);
          if (__builtin_expect(!all, 0)) st.mask(w, r, x[u], t8);
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          high[n] = st.highest(x[0][n]);
#pragma unroll
          for (int u = 1; u < kUnits; ++u) high[n] = larger(high[n], st.highest(x[u][n]));
          high[n] *= scale;
        }
        st.raise(high);
#pragma unroll
        for (int u = 0; u < kUnits; ++u) {
          bf16x8 p[1][NT];
          st.weigh(scale, x[u], p);
#pragma unroll
          for (int j = 0; j < DV; ++j) st.add(j, as_bf16(at[64 * (S::kV + u * DV + j)]), p);
        }
      }
      lds_barrier();   // the next tile of rows writes where these tokens are
      if (__builtin_expect(lds_odd[turn % 2] == turn, 0)) st.add_odd(w, r, from, to, kTokens, [&](int j, int i) { return 64 * (j / 4) + 16 * g + 4 * i + j % 4; });

      // lane (m, g) has elements 64 b + 16 g + 4 i + j of row m in acc[4 b + j][i]
      const AttentionArgs a = args_again();
      const uint32_t q_heads = a.cache.heads * a.group;
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const uint32_t row = r0 + 16 * n + m;
        const float total = st.total(n);
        if (row >= w.rows) continue;
        const uint32_t h = w.head * a.group + row % a.group;
        const uint64_t out_row = (uint64_t)(uint32_t)(w.s.start + (int)(row / a.group));
        if (w.whole) {
          const float f = one_over(total);
          uint8_t* to = a.out + out_row * a.out_stride + 2 * ((uint64_t)h * D + 16 * g);
#pragma unroll
          for (int b = 0; b < D / 64; ++b) {
            u32x4 o[2];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              o[i / 2][i % 2 * 2] = bf16_pair(st.acc[n][4 * b][i] * f, st.acc[n][4 * b + 1][i] * f);
              o[i / 2][i % 2 * 2 + 1] = bf16_pair(st.acc[n][4 * b + 2][i] * f, st.acc[n][4 * b + 3][i] * f);
            }
            *reinterpret_cast<u32x4*>(to + 128 * b) = o[0];
            *reinterpret_cast<u32x4*>(to + 128 * b + 16) = o[1];
          }
          if (g == 0 && a.lse) a.lse[out_row * q_heads + h] = lse_of(st.top[n], total);
        } else {
          const uint64_t place = w.place(a, 0, wave * 16 * NT + 16 * n + m);
          float* to = a.part_out + place * D + 16 * g;
#pragma unroll
          for (int b = 0; b < D / 64; ++b)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              *reinterpret_cast<f32x4*>(to + 64 * b + 4 * i) = f32x4{st.acc[n][4 * b][i], st.acc[n][4 * b + 1][i], st.acc[n][4 * b + 2][i], st.acc[n][4 * b + 3][i]};
          if (g == 0) {
            a.part_stat[2 * place] = st.top[n];
            a.part_stat[2 * place + 1] = total;
          }
        }
      }
    } while (w.more_rows());
  } while (w.next(lane));
}

// The parts of a sequence together.  D / 4 threads have a row and query head, four elements each: where the parts are few, as many rows
// as that leaves room for go through a workgroup at a time, otherwise all its threads take every (1024 / D)-th part of one.  Bound by
// latency: the blocks' count, the statistics and the parts are asked for one behind the other, 4 to 6 us; 15 us for the 32768 rows of 64 drafts
// of 16 sequences, some 50 MB of parts.  (Up to 48 parts sixteen at a time instead of by all threads: 4 and 52 rows of sequences of 1000 to 2000 tokens 1 us
// slower; four parts asked for as sixteen: 16 sequences of 4000 tokens under 256 rows 121 us a call, 109 so.  Four waves per SIMD: with a few
// registers too many for that 17 us where it takes 15.)
constexpr uint32_t kVeryFewParts = 4, kFewParts = 16;
template <int D>
__global__ void __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(4))) attention_join_kernel(AttentionArgs a) {
  constexpr uint32_t kAcross = D / 4, kDown = kThreads / kAcross;
  __shared__ f32x4 lds_out[kThreads];
  __shared__ float lds_sum[kDown], lds_top[kWaves];
  const uint32_t lane = threadIdx.x % 64, q_heads = a.cache.heads * a.group, groups = a.cache.heads / a.heads_across;
  Blocks b;
  Span mine;
  uint32_t front = 0;
  b.count(a, lane, mine);
  for (uint32_t at = 0; at < blockIdx.y; at += 64) {
    const uint32_t n = blocks_of(a, at ? spans_at(a, lane, at) : mine);
    front += wave_last(wave_incl_scan(at + lane < blockIdx.y ? n : 0));
  }
  const Span s = blockIdx.y < 64 ? Blocks::of_lane(mine, (int)blockIdx.y) : span_at(a, lane, blockIdx.y);
  const uint32_t blocks = blocks_of(a, s);
  if (blocks < 2 || (uint64_t)s.rows * a.group > a.most_rows) return;   // written already
  const uint32_t share0 = b.owner(front), n_parts = b.owner(front + blocks - 1) + 1 - share0;
  if (n_parts == 1) return;
  const uint32_t slot0 = b.begin(share0) < front ? 1 : 0;   // of the first part: behind another sequence's; the others are their workgroups' first
  const uint32_t across = threadIdx.x % kAcross, down = threadIdx.x / kAcross;
  const uint32_t outs = (uint32_t)s.rows * q_heads;
  const bool few = n_parts <= kFewParts;
  const uint32_t step = few ? kDown : 1;
  for (uint32_t u0 = blockIdx.x * step; u0 < outs; u0 += gridDim.x * step) {
    const uint32_t u = min(u0 + (few ? down : 0), outs - 1);
    const uint64_t out_row = (uint64_t)(uint32_t)(s.start + (int)(u / q_heads)), h = u % q_heads;
    const uint32_t head = (uint32_t)h / a.group, r = u / q_heads * a.group + (uint32_t)h % a.group, tile = r / a.tile_rows;
    const auto place = [&](uint32_t p) {
      const uint32_t unit = (share0 + p) * groups + head / a.heads_across;
      const uint64_t wg = ((uint64_t)(unit / 8) * a.row_tiles + tile) * 8 + unit % 8;
      return ((wg * 2 + (p ? 0 : slot0)) * a.heads_across + head % a.heads_across) * a.kept + r % a.tile_rows;
    };
    float high = kLowest, total = 0.0f;
    f32x4 o = {0, 0, 0, 0};
    if (few) {
      const auto add_parts = [&](auto most, uint32_t p0) {
        constexpr uint32_t N = decltype(most)::value;
        f32x4 x[N];
        float top[N], sum[N];
#pragma unroll
        for (uint32_t p = 0; p < N; ++p) {   // (the last one again where there are no more: a load behind a condition would wait for those before it)
          const uint64_t at = place(min(p0 + p, n_parts - 1));
          x[p] = *reinterpret_cast<const f32x4*>(a.part_out + at * D + 4 * across);
          top[p] = a.part_stat[2 * at];
          sum[p] = a.part_stat[2 * at + 1];
        }
        float now = high;
#pragma unroll
        for (uint32_t p = 0; p < N; ++p) now = fmaxf(now, top[p]);
        const float less = __builtin_amdgcn_exp2f(high - now);
        high = now;
        total *= less;
        o *= less;
#pragma unroll
        for (uint32_t p = 0; p < N; ++p) {
          if (p0 + p < n_parts) {
            const float f = __builtin_amdgcn_exp2f(top[p] - high);
            total += f * sum[p];
            o += f * x[p];
          }
        }
      };
      if (n_parts <= kVeryFewParts) {
        add_parts(std::integral_constant<uint32_t, kVeryFewParts>(), 0);
      } else {
        // (as a loop, though it runs once: straight, a call of one token over 777 takes 12.4 us instead of 10.8)
        for (uint32_t p0 = 0; p0 < n_parts; p0 += kFewParts) add_parts(std::integral_constant<uint32_t, kFewParts>(), p0);
      }
    } else {
      for (uint32_t p = threadIdx.x; p < n_parts; p += kThreads) high = fmaxf(high, a.part_stat[2 * place(p)]);
#pragma unroll
      for (int k = 32; k > 0; k /= 2) high = fmaxf(high, __shfl_xor(high, k));
      __syncthreads();   // (the row before this one has been read)
      if (lane == 0) lds_top[threadIdx.x / 64] = high;
      __syncthreads();
#pragma unroll
      for (int k = 0; k < kWaves; ++k) high = fmaxf(high, lds_top[k]);
#pragma unroll 4
      for (uint32_t p = down; p < n_parts; p += kDown) {
        const uint64_t at = place(p);
        const f32x4 x = *reinterpret_cast<const f32x4*>(a.part_out + at * D + 4 * across);
        const float f = __builtin_amdgcn_exp2f(a.part_stat[2 * at] - high);
        total += f * a.part_stat[2 * at + 1];
        o += f * x;
      }
      lds_out[threadIdx.x] = o;
      if (across == 0) lds_sum[down] = total;
      __syncthreads();
      if (down != 0) continue;
      for (uint32_t k = 1; k < kDown; ++k) {
        o += lds_out[k * kAcross + across];
        total += lds_sum[k];
      }
    }
    const float f = one_over(total);
    *reinterpret_cast<u32x2*>(a.out + out_row * a.out_stride + 2 * (h * D + 4 * across)) = u32x2{bf16_pair(o[0] * f, o[1] * f), bf16_pair(o[2] * f, o[3] * f)};
    if (across == 0 && a.lse) a.lse[out_row * q_heads + h] = lse_of(high, total);
  }
}

#endif  // SPLITZIP_ATTENTION_HPP
