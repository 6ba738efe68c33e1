// SplitZip for MI355X: a step's projections on their way to the cache -- the heads of Q and K normed and turned by their rows' positions, K and V
// written into the cache, Q into the tensor that attention takes.  Part of the single translation unit cache.hip (included inside
// its anonymous namespace, behind cache.hpp).
//
// A head x of D elements, of a row at position p:
//   y_d = x_d / sqrt(mean of x^2 + eps) * (w_d + offset)             (norms; without weights w_d + offset is 1)
//   (y_a, y_b) -> s (y_a cos t - y_b sin t, y_b cos t + y_a sin t),  t = p f_i,  i = 0 .. R / 2 - 1
// with (a, b) = (2 i, 2 i + 1) or (i, i + R / 2) for the first R elements; the others stay as they are.  All in 32 bits, and rounded
// once, to what is written; t in 64 bits, in turns, of which the whole ones are dropped before sine and cosine: positions go up to 2^30,
// where 32 bits of an angle would leave nothing of it.
//
// A row's sines and cosines are the same for all of its heads: a workgroup belongs to one row at a time, its first R / 2 threads make an angle
// each while the heads' words are on their way, and all lanes read their eight elements' from LDS.  D / 8 lanes take a head, eight elements each, as in
// cache_write_kernel; what a lane's elements are turned with lies in another lane of the same head.
#ifndef SPLITZIP_APPEND_HPP
#define SPLITZIP_APPEND_HPP

struct AppendArgs {
  Cache cache;
  Seqs seqs;
  const uint8_t *q, *k, *v;
  uint8_t *q_out, *k_out;                                          // k_out: or null
  uint64_t q_stride, k_stride, v_stride, q_out_stride, k_out_stride;   // bytes from row to row
  const float* freqs;
  const void *q_weight, *k_weight;                                 // or null
  const int32_t* positions;                                        // [n_rows] or null: base + row
  float scaling, eps, weight_offset;
  uint32_t q_heads, rotary;
  uint32_t interleaved, norm, weights_f32;
  uint32_t chunks;                                                 // workgroups of a row
};

// eight elements of a lane, in 32 bits, as words of the cache, and the byte of the lane's scale
template <int KIND, int D>
__device__ inline Lane8<KIND> quantised(const float (&y)[8], int& byte) {
  if constexpr (KIND == SPLITZIP_BF16) {
    return u32x4{bf16_pair(y[0], y[1]), bf16_pair(y[2], y[3]), bf16_pair(y[4], y[5]), bf16_pair(y[6], y[7])};
  } else {
    uint32_t m = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t x = __float_as_uint(y[e]) & 0x7fffffffu;
      m = max(m, KIND == SPLITZIP_FP4_E2M1 || x < 0x7f800000u ? x : 0u);
    }
    m = largest_of_group<KIND, D>(m);
    byte = KIND == SPLITZIP_FP4_E2M1 && m >= 0x7f800000u ? 255 : scale_byte<KIND>(m);
    if constexpr (KIND == SPLITZIP_FP4_E2M1) return to_fp4(y, byte);
    else return to_fp8<KIND>(y, byte);
  }
}

// weights of a lane's eight elements, the offset added
__device__ inline void load_weights(const AppendArgs& a, const void* at, uint32_t lane, float (&w)[8]) {
  if (!at) {
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = 1.0f;
    return;
  }
  if (a.weights_f32) {
    const f32x4 lo = reinterpret_cast<const f32x4*>(at)[2 * lane], hi = reinterpret_cast<const f32x4*>(at)[2 * lane + 1];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      w[e] = lo[e];
      w[4 + e] = hi[e];
    }
  } else {
    floats_of(reinterpret_cast<const u32x4*>(at)[lane], w);
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) w[e] += a.weight_offset;
}

// N: heads of each lane at a time
constexpr int kAppendHeads = 4;
template <int KIND, int D, int N>
__global__ void __launch_bounds__(kThreads) cache_append_kernel(AppendArgs a) {
  constexpr uint32_t kLanes = D / 8, kHeads = kThreads / kLanes;
  __shared__ float turns[2][2][D / 2];   // of the even and of the odd rows that the workgroup takes: cosines, sines
  const uint32_t lane = threadIdx.x % kLanes, half = a.rotary / 2;
  const Seq s = seq_at(a.seqs, blockIdx.y);
  const Pages pages(a.cache, a.seqs, blockIdx.y);
  const uint32_t heads = a.q_heads + 2 * a.cache.heads;   // those of Q, of K, of V
  const uint32_t first = blockIdx.x % a.chunks * N * kHeads + threadIdx.x / kLanes;
  const uint32_t step = gridDim.x / a.chunks;
  float q_weight[8], k_weight[8];
  if (a.norm) {
    load_weights(a, a.q_weight, lane, q_weight);
    load_weights(a, a.k_weight, lane, k_weight);
  }
  uint32_t parity = 0;
  for (uint32_t i = blockIdx.x / a.chunks; i < (uint32_t)s.rows; i += step, parity ^= 1) {
    const uint64_t row = (uint32_t)s.start + i;
    const int token = s.base + (int)i;
    u32x4 x[N];
#pragma unroll
    for (int n = 0; n < N; ++n) {   // (the last head once more where there are no more: no load stands behind a condition)
      const uint32_t h = min(first + n * kHeads, heads - 1);
      const uint8_t* const at = h < a.q_heads ? a.q + row * a.q_stride + 2 * (uint64_t)h * D
                                : h < a.q_heads + a.cache.heads ? a.k + row * a.k_stride + 2 * (uint64_t)(h - a.q_heads) * D
                                                                : a.v + row * a.v_stride + 2 * (uint64_t)(h - a.q_heads - a.cache.heads) * D;
      x[n] = *reinterpret_cast<const u32x4*>(as_global(at) + 16 * lane);
    }
    const uint32_t page = pages.page((uint32_t)max(token, 0)), place = pages.place((uint32_t)max(token, 0));
    if (threadIdx.x < half) {
      const int position = a.positions ? a.positions[row] : token;
      const double turn = (double)position * ((double)a.freqs[threadIdx.x] * 0.15915494309189533577);
      float sine, cosine;
      sincospif(2.0f * (float)(turn - rint(turn)), &sine, &cosine);
      turns[parity][0][threadIdx.x] = cosine * a.scaling;
      turns[parity][1][threadIdx.x] = sine * a.scaling;
    }
    lds_barrier();   // (a place is written again by the second row after this one, a barrier on)
    // the lane's elements times `same`, the others of their pairs times `other`
    float same[8], other[8];
    const bool turned = 8 * lane < a.rotary;
    if (turned) {
      if (a.interleaved) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float c = turns[parity][0][4 * lane + e], sn = turns[parity][1][4 * lane + e];
          same[2 * e] = same[2 * e + 1] = c;
          other[2 * e] = -sn;
          other[2 * e + 1] = sn;
        }
      } else {
        const bool upper = 8 * lane >= half;
        const uint32_t f = 8 * lane - (upper ? half : 0);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          same[e] = turns[parity][0][f + e];
          other[e] = upper ? turns[parity][1][f + e] : -turns[parity][1][f + e];
        }
      }
    }
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const uint32_t h = first + n * kHeads;
      if (h >= heads) continue;
      const bool of_q = h < a.q_heads, of_k = !of_q && h < a.q_heads + a.cache.heads;
      float y[8];
      floats_of(x[n], y);
      if (of_q || of_k) {
        if (a.norm) {
          float sum = 0.0f;
#pragma unroll
          for (int e = 0; e < 8; ++e) sum += y[e] * y[e];
#pragma unroll
          for (uint32_t o = kLanes / 2; o > 0; o /= 2) sum += __shfl_xor(sum, (int)o);
          const float over = rsqrtf(sum * (1.0f / D) + a.eps);
#pragma unroll
          for (int e = 0; e < 8; ++e) y[e] = y[e] * over * (of_q ? q_weight[e] : k_weight[e]);
        }
        if (a.rotary) {
          float z[8];
          if (a.interleaved) {
#pragma unroll
            for (int e = 0; e < 8; ++e) z[e] = y[e ^ 1];
          } else {
            const int from = (int)(threadIdx.x + (8 * lane < half ? half / 8 : turned ? 0u - half / 8 : 0u));
#pragma unroll
            for (int e = 0; e < 8; ++e) z[e] = __shfl(y[e], from);
          }
          if (turned) {
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = y[e] * same[e] + z[e] * other[e];
          }
        }
      }
      if (of_q) {
        int none;
        *reinterpret_cast<u32x4*>(a.q_out + row * a.q_out_stride + 2 * ((uint64_t)h * D + 8 * lane)) = quantised<SPLITZIP_BF16, D>(y, none);
        continue;
      }
      const uint32_t head = h - a.q_heads - (of_k ? 0 : a.cache.heads);
      if (of_k && a.k_out) {
        int none;
        *reinterpret_cast<u32x4*>(a.k_out + row * a.k_out_stride + 2 * ((uint64_t)head * D + 8 * lane)) = quantised<SPLITZIP_BF16, D>(y, none);
      }
      if (token < 0) continue;
      int byte = 0;
      const Lane8<KIND> words = quantised<KIND, D>(y, byte);
      const uint64_t at = token_offset(a.cache, page, place) + head * a.cache.head_stride + lane * kBits<KIND>;
      *reinterpret_cast<Lane8<KIND>*>((of_k ? a.cache.k : a.cache.v) + at) = words;
      if constexpr (KIND != SPLITZIP_BF16) {
        if (has_scale<KIND, D>(lane)) (of_k ? a.cache.k_scales : a.cache.v_scales)[scale_offset(a.cache, page, place, scale_row<KIND, D>(head, lane))] = (uint8_t)byte;
      }
    }
  }
}

#endif  // SPLITZIP_APPEND_HPP
