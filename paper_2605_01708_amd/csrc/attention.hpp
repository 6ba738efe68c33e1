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
// Both operands come straight from memory into registers, every byte once: K as rows, V as eight tokens times D / 16
// elements per lane, transposed in registers by byte permutes.
//
// Statistics, outputs and the sums over waves and over the parts of a long sequence are held in 32 bits.  P goes into the second
// product as BF16, as V does (relative error 2^-9 per token, as that of the BF16 result); the sum of P is taken before that rounding.
#ifndef SPLITZIP_ATTENTION_HPP
#define SPLITZIP_ATTENTION_HPP

constexpr uint32_t kStep = 32;          // tokens of a wave at a time
constexpr float kLowest = -3.0e38f;     // the running maximum before the first score (finite: differences stay numbers)
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
  float* part_out;                   // [n_rows][q_heads][parts][D]
  float* part_stat;                  // [n_rows][q_heads][parts][2]: maximum (of log2), sum
  float scale, softcap;
  uint32_t tree_words, window;       // window 0: none
  uint32_t group, parts, part_tokens, row_tiles;
};

__device__ inline int position_of(const AttentionArgs& a, const Seq& s, int i) {
  return a.positions ? a.positions[s.start + i] : s.base + i;
}

// The first token that any row of the sequence may see, a multiple of 32: with a window, the one that the row at the lowest
// position sees.  The parts of a sequence count from it.
__device__ inline int first_token(const AttentionArgs& a, const Seq& s, uint32_t lane) {
  if (!a.window) return 0;
  int low = s.base;   // without positions: the first row's
  if (a.positions) {
    low = 0x7fffffff;
    for (int i = (int)lane; i < s.rows; i += 64) low = min(low, position_of(a, s, i));
#pragma unroll
    for (int o = 32; o > 0; o /= 2) low = min(low, __shfl_xor(low, o));
  }
  const int64_t first = (int64_t)low - (int64_t)a.window + 1;
  const int64_t most = max(min(s.base, s.len), 0);   // drafted tokens lie where their positions say, not where they are stored
  return (int)(max(min(first, most), (int64_t)0) & ~(int64_t)(kStep - 1));
}

__device__ inline uint32_t parts_of(const AttentionArgs& a, const Seq& s, int first) {
  const uint32_t n = ((uint32_t)(s.len - first) + a.part_tokens - 1) / a.part_tokens;
  return min(max(n, 1u), a.parts);
}

// the scores' way into the exponent of two
__device__ inline float shaped(const AttentionArgs& a, float x, float slope_log2, float far) {
  if (a.softcap > 0.0f) {
    // tanh(y) = 1 - 2 / (1 + e^2y): its absolute error of 1e-7 times the cap is one of the exponent
    const float e = __builtin_amdgcn_exp2f(x * (2.0f * kLog2e / a.softcap));
    x = a.softcap - (2.0f * a.softcap) * __builtin_amdgcn_rcpf(1.0f + e);
  }
  return x * kLog2e - slope_log2 * far;
}

__device__ inline f32x4 mfma(const bf16x8& x, const bf16x8& y, const f32x4& c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, y, c, 0, 0, 0); }

template <int KIND, int D, int NT>
__global__ void __launch_bounds__(kThreads) attention_kernel(AttentionArgs a) {
  constexpr int ES = KIND == SPLITZIP_BF16 ? 2 : 1;
  constexpr int KS = D / 32;     // steps of the first product
  constexpr int DV = D / 16;     // elements of V per lane and token, and tiles of the second product
  constexpr int kRow = D + 4;    // floats of a row in LDS
  __shared__ float lds_out[kWaves * 16 * kRow];
  __shared__ float lds_stat[kWaves][16][2];
  const uint32_t lane = threadIdx.x % 64, wave = threadIdx.x / 64, m = lane % 16, g = lane / 16;

  // workgroups of the same (part, sequence, head) lie 8 apart, on the same XCD
  const uint32_t of = blockIdx.x / 8 / a.row_tiles, tile0 = blockIdx.x / 8 % a.row_tiles;
  const uint32_t unit = of * 8 + blockIdx.x % 8;
  const uint32_t head = unit % a.cache.heads, seq = unit / a.cache.heads % a.seqs.n_seqs, part = unit / a.cache.heads / a.seqs.n_seqs;
  if (part >= a.parts) return;
  const Seq s = seq_at(a.seqs, seq);
  const int first = first_token(a, s, lane);
  const uint32_t n_parts = parts_of(a, s, first);
  if (part >= n_parts) return;
  const int begin = first + (int)(part * a.part_tokens);
  const int end = part + 1 < n_parts ? begin + (int)a.part_tokens : s.len;   // the last one goes on to the end
  const uint32_t rows = (uint32_t)s.rows * a.group, q_heads = a.cache.heads * a.group;

  for (uint32_t tile = tile0; tile * 16 * NT < rows; tile += a.row_tiles) {
    // the lane's rows, and their operand of the first product
    int row[NT], pos[NT];
    float slope[NT];
    bf16x8 q[NT][KS];
    int64_t low_edge = -0x7fffffffffffffff;   // tokens up to here may be out of a row's window
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const uint32_t r = (tile * NT + n) * 16 + m;
      const bool have = r < rows;
      row[n] = have ? (int)(r / a.group) : -1;
      const uint32_t h = head * a.group + (have ? r % a.group : 0);
      pos[n] = have ? position_of(a, s, row[n]) : 0;
      slope[n] = a.slopes ? a.slopes[h] * kLog2e : 0.0f;
      if (have && a.window) low_edge = max(low_edge, (int64_t)pos[n] - (int64_t)a.window);
      const uint8_t* at = a.q + (uint64_t)(uint32_t)(s.start + max(row[n], 0)) * a.q_stride + 2 * (uint64_t)h * D;
#pragma unroll
      for (int t = 0; t < KS; ++t) {
        // FP8 rows are loaded 16 bytes, two steps, at a time: the same order here
        const uint32_t d = KIND == SPLITZIP_BF16 ? 32 * t + 8 * g : 64 * (t / 2) + 16 * g + 8 * (t % 2);
        u32x4 w = {0, 0, 0, 0};
        if (have) w = *reinterpret_cast<const u32x4*>(at + 2 * d);
        q[n][t] = __builtin_bit_cast(bf16x8, w);
      }
    }
    if (a.window) {
#pragma unroll
      for (int o = 8; o > 0; o /= 2) low_edge = max(low_edge, (int64_t)__shfl_xor((long long)low_edge, o));
    }

    f32x4 acc[NT][DV];
    float top[NT], sum[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      top[n] = kLowest;
      sum[n] = 0.0f;
#pragma unroll
      for (int j = 0; j < DV; ++j) acc[n][j] = f32x4{0, 0, 0, 0};
    }

    for (int t0 = begin + (int)(wave * kStep); t0 < end; t0 += (int)(kWaves * kStep)) {
      // tokens 8 (m / 4) + .. for K, 8 g + .. for V; those behind the sequence's end are read at its last eight
      const uint32_t last8 = (uint32_t)(s.len - 1) & ~7u;
      const uint32_t k8 = min((uint32_t)t0 + 8 * (m / 4), last8), v8 = min((uint32_t)t0 + 8 * g, last8);
      const uint32_t k_page = page_of_token(a.cache, a.seqs, seq, k8), k_place = place_of_token(a.cache, a.seqs, k8) + m % 4;
      const uint32_t v_page = page_of_token(a.cache, a.seqs, seq, v8), v_place = place_of_token(a.cache, a.seqs, v8);
      const uint8_t* k_at = a.cache.k + word_offset(a.cache, k_page, k_place, head);
      const uint8_t* v_at = a.cache.v + word_offset(a.cache, v_page, v_place, head);

      f32x4 x[NT][2];
#pragma unroll
      for (int n = 0; n < NT; ++n) x[n][0] = x[n][1] = f32x4{0, 0, 0, 0};
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const uint8_t* at = k_at + 4 * b * a.cache.token_stride;
        if constexpr (KIND == SPLITZIP_BF16) {
#pragma unroll
          for (int t = 0; t < KS; ++t) {
            const bf16x8 k = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(at + 2 * (32 * t + 8 * g)));
#pragma unroll
            for (int n = 0; n < NT; ++n) x[n][b] = mfma(k, q[n][t], x[n][b]);
          }
        } else {
#pragma unroll
          for (int t = 0; t < KS; t += 2) {
            const u32x4 w = *reinterpret_cast<const u32x4*>(at + 32 * t + 16 * g);
#pragma unroll
            for (int u = 0; u < 2; ++u) {
              const u32x4 f = {fp8_pair_to_bf16<KIND, false>(w[2 * u]), fp8_pair_to_bf16<KIND, true>(w[2 * u]),
                               fp8_pair_to_bf16<KIND, false>(w[2 * u + 1]), fp8_pair_to_bf16<KIND, true>(w[2 * u + 1])};
#pragma unroll
              for (int n = 0; n < NT; ++n) x[n][b] = mfma(__builtin_bit_cast(bf16x8, f), q[n][t + u], x[n][b]);
            }
          }
        }
      }
      // V: DV elements of each of the eight tokens, as BF16; vt[j]: element j of all eight
      u32x4 vt[DV];
      {
        uint32_t w[8][DV / 2];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const uint8_t* at = v_at + e * a.cache.token_stride + ES * DV * m;
          if constexpr (KIND == SPLITZIP_BF16) {
            __builtin_memcpy(w[e], __builtin_assume_aligned(at, 2 * DV < 16 ? 2 * DV : 16), 2 * DV);
          } else {
            uint32_t raw[DV / 4];
            __builtin_memcpy(raw, __builtin_assume_aligned(at, DV < 16 ? DV : 16), DV);
#pragma unroll
            for (int i = 0; i < DV / 4; ++i) {
              w[e][2 * i] = fp8_pair_to_bf16<KIND, false>(raw[i]);
              w[e][2 * i + 1] = fp8_pair_to_bf16<KIND, true>(raw[i]);
            }
          }
        }
#pragma unroll
        for (int j = 0; j < DV; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i) vt[j][i] = byte_perm(w[2 * i + 1][j / 2], w[2 * i][j / 2], j % 2 ? 0x07060302u : 0x05040100u);
      }
      // the scales of the lane's eight tokens
      u32x2 k_scales = {0, 0}, v_scales = {0, 0};
      if constexpr (KIND != SPLITZIP_BF16) {
        const uint64_t scale = scale_offset(a.cache, a.seqs, v_page, v_place, head);
        k_scales = *reinterpret_cast<const u32x2*>(a.cache.k_scales + scale);
        v_scales = *reinterpret_cast<const u32x2*>(a.cache.v_scales + scale);
      }

      const bool all = t0 + (int)kStep <= min(s.base, s.len) && (int64_t)t0 > low_edge;   // every row sees every token
      uint32_t seen[NT];   // bit e: the lane's row sees the lane's token e
#pragma unroll
      for (int n = 0; n < NT; ++n) seen[n] = 0xffu;
      if (!all) {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          seen[n] = 0;
          for (int e = 0; e < 8; ++e) {
            const int t = t0 + (int)(8 * g) + e, j = t - s.base;
            bool ok = row[n] >= 0 && t < s.len;
            if (ok && j >= 0) {
              if (a.tree) ok = (uint32_t)j / 64 < a.tree_words && (a.tree[(uint64_t)(uint32_t)(s.start + row[n]) * a.tree_words + (uint32_t)j / 64] >> (j % 64) & 1);
              else ok = j <= row[n];
            }
            if (ok && a.window) ok = (int64_t)pos[n] - (int64_t)(j >= 0 ? position_of(a, s, j) : t) < (int64_t)a.window;
            seen[n] |= (uint32_t)ok << e;
          }
        }
      }

      bf16x8 p[NT];
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        float y[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float v = x[n][e / 4][e % 4] * a.scale;
          if constexpr (KIND != SPLITZIP_BF16) v *= two_to((int)(k_scales[e / 4] >> (8 * (e % 4)) & 0xffu));
          float far = 0.0f;
          if (a.slopes) {
            const int t = t0 + (int)(8 * g) + e, j = t - s.base;
            const int at = j >= 0 && t < s.len ? position_of(a, s, j) : t;
            far = (float)(pos[n] - at);
          }
          v = shaped(a, v, slope[n], far);
          y[e] = seen[n] >> e & 1 ? v : -__builtin_inff();
        }
        float high = y[0];
#pragma unroll
        for (int e = 1; e < 8; ++e) high = fmaxf(high, y[e]);
        high = fmaxf(high, __shfl_xor(high, 16));
        high = fmaxf(high, __shfl_xor(high, 32));
        const float now = fmaxf(top[n], high), less = __builtin_amdgcn_exp2f(top[n] - now);
        top[n] = now;
        sum[n] *= less;
#pragma unroll
        for (int j = 0; j < DV; ++j) acc[n][j] *= less;
        float w[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          w[e] = __builtin_amdgcn_exp2f(y[e] - now);
          sum[n] += w[e];
          if constexpr (KIND != SPLITZIP_BF16) w[e] *= two_to((int)(v_scales[e / 4] >> (8 * (e % 4)) & 0xffu));
          if (!(seen[n] >> e & 1)) w[e] = 0.0f;   // whatever a token's scale holds that the row does not see
        }
        const u32x4 packed = {bf16_pair(w[0], w[1]), bf16_pair(w[2], w[3]), bf16_pair(w[4], w[5]), bf16_pair(w[6], w[7])};
        p[n] = __builtin_bit_cast(bf16x8, packed);
      }

      if (!all) {
        // A token that some row does not see may hold anything, and 0 times an infinity or a NaN is no 0: tokens with such
        // words are taken out of the product, and added one by one to the rows that see them.
        const int t8 = t0 + (int)(8 * g);
        uint32_t odd = 0;   // bit e: token e of the lane's eight has such a word in the lane's columns
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          bool any = false;
#pragma unroll
          for (int j = 0; j < DV; ++j) any |= (vt[j][e / 2] >> (16 * (e % 2)) & 0x7f80u) == 0x7f80u;
          odd |= (uint32_t)any << e;
        }
#pragma unroll
        for (int o = 8; o > 0; o /= 2) odd |= (uint32_t)__shfl_xor((int)odd, o);   // all columns of the token
        uint32_t behind = 0;   // tokens behind the end: nobody's
#pragma unroll
        for (int e = 0; e < 8; ++e) behind |= (uint32_t)(t8 + e >= s.len) << e;
        uint32_t keep[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t out2 = (odd | behind) >> (2 * i);
          keep[i] = (out2 & 1 ? 0u : 0xffffu) | (out2 & 2 ? 0u : 0xffff0000u);
        }
        const uint32_t alone = odd & ~behind;
        if (__ballot(alone != 0)) {
          for (uint32_t t = 0; t < kStep; ++t) {
            if (!((uint32_t)__builtin_amdgcn_readlane((int)alone, (int)(t / 8 * 16)) >> (t % 8) & 1)) continue;
            u32x4 just;
#pragma unroll
            for (int i = 0; i < 4; ++i) just[i] = g == t / 8 && i == (int)(t % 8 / 2) ? (t % 2 ? 0xffff0000u : 0xffffu) : 0u;
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              const bool mine = (uint32_t)__shfl((int)seen[n], (int)(t / 8 * 16 + m)) >> (t % 8) & 1;
              // (the row's own weight alone: another token's 0 times this one's infinity is a NaN as well)
              const bf16x8 only = __builtin_bit_cast(bf16x8, __builtin_bit_cast(u32x4, p[n]) & just);
#pragma unroll
              for (int j = 0; j < DV; ++j) {
                const f32x4 c = mfma(__builtin_bit_cast(bf16x8, vt[j] & just), only, f32x4{0, 0, 0, 0});
                if (mine) acc[n][j] += c;
              }
            }
          }
        }
#pragma unroll
        for (int j = 0; j < DV; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i) vt[j][i] &= keep[i];
      }
#pragma unroll
      for (int j = 0; j < DV; ++j)
#pragma unroll
        for (int n = 0; n < NT; ++n) acc[n][j] = mfma(__builtin_bit_cast(bf16x8, vt[j]), p[n], acc[n][j]);
    }

    // the four waves' parts of the tokens together
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      sum[n] += __shfl_xor(sum[n], 16);
      sum[n] += __shfl_xor(sum[n], 32);
      __syncthreads();
      if (g == 0) {
        lds_stat[wave][m][0] = top[n];
        lds_stat[wave][m][1] = sum[n];
      }
      // lane (m, g) has elements 4 DV g + DV i + j of row m in acc[j][i]
      float* mine = lds_out + (wave * 16 + m) * kRow + 4 * DV * g;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < DV; j += 4) *reinterpret_cast<f32x4*>(mine + DV * i + j) = f32x4{acc[n][j][i], acc[n][j + 1][i], acc[n][j + 2][i], acc[n][j + 3][i]};
      __syncthreads();
      const uint32_t r = threadIdx.x / 16, c = threadIdx.x % 16, at = (tile * NT + n) * 16 + r;
      if (at < rows) {
        float high = lds_stat[0][r][0], total = 0.0f, o[DV];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) high = fmaxf(high, lds_stat[w][r][0]);
#pragma unroll
        for (int j = 0; j < DV; ++j) o[j] = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
          const float f = __builtin_amdgcn_exp2f(lds_stat[w][r][0] - high);
          total += f * lds_stat[w][r][1];
#pragma unroll
          for (int j = 0; j < DV; ++j) o[j] += f * lds_out[(w * 16 + r) * kRow + DV * c + j];
        }
        const uint32_t i = at / a.group, h = head * a.group + at % a.group;
        const uint64_t out_row = (uint64_t)(uint32_t)(s.start + (int)i);
        if (n_parts == 1) {
          const float f = total != 0.0f ? 1.0f / total : 0.0f;   // (a NaN is no 0)
          uint8_t* to = a.out + out_row * a.out_stride + 2 * ((uint64_t)h * D + DV * c);
#pragma unroll
          for (int j = 0; j < DV; j += 2) *reinterpret_cast<uint32_t*>(to + 2 * j) = bf16_pair(o[j] * f, o[j + 1] * f);
          if (c == 0 && a.lse) a.lse[out_row * q_heads + h] = total != 0.0f ? (high + __builtin_amdgcn_logf(total)) * kLn2 : -__builtin_inff();
        } else {
          const uint64_t place = (out_row * q_heads + h) * a.parts + part;
#pragma unroll
          for (int j = 0; j < DV; j += 4) *reinterpret_cast<f32x4*>(a.part_out + place * D + DV * c + j) = f32x4{o[j], o[j + 1], o[j + 2], o[j + 3]};
          if (c == 0) {
            a.part_stat[2 * place] = high;
            a.part_stat[2 * place + 1] = total;
          }
        }
      }
    }
  }
}

// The parts of a sequence together: a wave per row and query head.
template <int D>
__global__ void __launch_bounds__(kThreads) attention_join_kernel(AttentionArgs a) {
  constexpr int PER = D / 64;
  const uint32_t lane = threadIdx.x % 64, q_heads = a.cache.heads * a.group;
  const Seq s = seq_at(a.seqs, blockIdx.y);
  const uint32_t n_parts = parts_of(a, s, first_token(a, s, lane));
  if (n_parts == 1) return;   // written already
  for (uint32_t u = blockIdx.x * kWaves + threadIdx.x / 64; u < (uint32_t)s.rows * q_heads; u += gridDim.x * kWaves) {
    const uint64_t out_row = (uint64_t)(uint32_t)(s.start + (int)(u / q_heads)), h = u % q_heads;
    const uint64_t place = (out_row * q_heads + h) * a.parts;
    float high = kLowest;
    for (uint32_t p = 0; p < n_parts; ++p) high = fmaxf(high, a.part_stat[2 * (place + p)]);
    float total = 0.0f, o[PER] = {};
    for (uint32_t p = 0; p < n_parts; ++p) {
      const float f = __builtin_amdgcn_exp2f(a.part_stat[2 * (place + p)] - high);
      total += f * a.part_stat[2 * (place + p) + 1];
#pragma unroll
      for (int j = 0; j < PER; ++j) o[j] += f * a.part_out[(place + p) * D + PER * lane + j];
    }
    const float f = total != 0.0f ? 1.0f / total : 0.0f;
    uint8_t* to = a.out + out_row * a.out_stride + 2 * (h * D + PER * lane);
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const __bf16 b = (__bf16)(o[j] * f);
      *reinterpret_cast<__bf16*>(to + 2 * j) = b;
    }
    if (lane == 0 && a.lse) a.lse[out_row * q_heads + h] = total != 0.0f ? (high + __builtin_amdgcn_logf(total)) * kLn2 : -__builtin_inff();
  }
}

#endif  // SPLITZIP_ATTENTION_HPP
