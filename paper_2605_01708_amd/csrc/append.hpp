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
// A row's sines and cosines are the same for all of its heads: a workgroup makes those of a few rows at a time, an angle per thread, and all
// lanes read their eight elements' from LDS.  D / 8 lanes take a head, eight elements each, as in cache_write_kernel; what a lane's elements
// are turned with lies in another lane of the same head.
//
// Bound by memory for long calls, by the launch for short ones.  16384 rows of 32 + 8 + 8 heads of 128 into E4M3, 369 MB: 68.3 us (5.4 TB/s; a plain
// copy of that mix of reads and writes 5.6); streamed loads alone 73.4, streamed stores alone 70.6, neither 73.0; workgroups: 6 per CU 74.6, 12 73.4,
// 24 70.2, 48 as it is, 96 68.4.  The next row's words are asked for before this one's are worked on, and a workgroup keeps its heads: the first form,
// a row at a time with all of its heads, took 123.  A workgroup's lanes hold 16 heads of 128: of fewer heads the others do the last one's work once more
// (42 sequences of 1660 rows, 4 + 2 heads of 128, E4M3: 78 us for 197 MB).
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
  uint32_t chunks, each;                                           // workgroups of a row; rows that one takes at a time
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

// A lane's eight elements turned; cosines and sines of the row, `half` each.
template <int D>
__device__ inline void turn(const AppendArgs& a, const float (*turns)[D / 2], uint32_t lane, uint32_t half, float (&y)[8]) {
  const bool turned = 8 * lane < a.rotary;
  if (a.interleaved) {
    const uint32_t f = turned ? 4 * lane : 0;
    const f32x4 c = *reinterpret_cast<const f32x4*>(turns[0] + f), s = *reinterpret_cast<const f32x4*>(turns[1] + f);
    if (!turned) return;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float u = y[2 * e], v = y[2 * e + 1];
      y[2 * e] = u * c[e] - v * s[e];
      y[2 * e + 1] = v * c[e] + u * s[e];
    }
    return;
  }
  const bool upper = 8 * lane >= half;
  float z[8];   // the pairs' other halves
  if (D == 128 && half == 64) {   // eight lanes on, in rows of sixteen
#pragma unroll
    for (int e = 0; e < 8; ++e) z[e] = __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(y[e]), 0x128, 0xf, 0xf, false));
  } else {
    const int from = (int)(threadIdx.x + (!upper ? half / 8 : turned ? 0u - half / 8 : 0u));
#pragma unroll
    for (int e = 0; e < 8; ++e) z[e] = __shfl(y[e], from);
  }
  const uint32_t f = turned ? 8 * lane - (upper ? half : 0) : 0;
  const f32x4 *const cs = reinterpret_cast<const f32x4*>(turns[0] + f), *const sn = reinterpret_cast<const f32x4*>(turns[1] + f);
  const f32x4 c[2] = {cs[0], cs[1]}, s[2] = {sn[0], sn[1]};
  if (!turned) return;
#pragma unroll
  for (int e = 0; e < 8; ++e) y[e] = y[e] * c[e / 4][e % 4] + z[e] * (upper ? s[e / 4][e % 4] : -s[e / 4][e % 4]);
}

template <int D>
constexpr uint32_t kAppendRows = 2 * kThreads / D;   // of which a workgroup makes the angles at a time: one per thread

template <int KIND, int D, bool STREAM>
__global__ void __launch_bounds__(kThreads) cache_append_kernel(AppendArgs a) {
  constexpr uint32_t kLanes = D / 8, kHeads = kThreads / kLanes;
  __shared__ __attribute__((aligned(16))) float turns[2][kAppendRows<D>][2][D / 2];   // of the even and of the odd times: of a row cosines, sines
  const uint32_t lane = threadIdx.x % kLanes, half = a.rotary / 2;
  const Seq s = seq_at(a.seqs, blockIdx.y);
  const Pages pages(a.cache, a.seqs, blockIdx.y);
  // the lane's head: one of Q, of K, of V (the last one once more where there are no more)
  const uint32_t kv = a.cache.heads, heads = a.q_heads + 2 * kv, chunk = blockIdx.x % a.chunks * kHeads, here = chunk + threadIdx.x / kLanes, h = min(here, heads - 1);
  const bool of_q = h < a.q_heads, of_k = !of_q && h < a.q_heads + kv, rotates = a.rotary && chunk < a.q_heads + kv;   // (rotates: one of the workgroup's)
  const uint32_t head = of_q ? h : h - a.q_heads - (of_k ? 0 : kv);
  const uint64_t stride = of_q ? a.q_stride : of_k ? a.k_stride : a.v_stride;
  const uint8_t* const from = as_global(of_q ? a.q : of_k ? a.k : a.v) + 2 * ((uint64_t)head * D + 8 * lane);
  float weight[8];
  if (a.norm && (of_q || of_k)) load_weights(a, of_q ? a.q_weight : a.k_weight, lane, weight);
  const uint32_t first = blockIdx.x / a.chunks * a.each, step = gridDim.x / a.chunks * a.each, rows = (uint32_t)s.rows;
  const auto load = [&](uint32_t i) { return ld_row<STREAM, u32x4>(from + (uint64_t)((uint32_t)s.start + i) * stride); };
  u32x4 next = {0, 0, 0, 0};
  if (first < rows) next = load(first);
  uint32_t parity = 0;
  for (uint32_t i0 = first; i0 < rows; i0 += step, parity ^= 1) {
    if (rotates) {
      const uint32_t r = threadIdx.x / (D / 2), f = threadIdx.x % (D / 2);
      if (r < a.each && i0 + r < rows && f < half) {
        const int position = a.positions ? a.positions[(uint32_t)s.start + i0 + r] : s.base + (int)(i0 + r);
        const double turn = (double)position * ((double)a.freqs[f] * 0.15915494309189533577);
        float sine, cosine;
        sincospif(2.0f * (float)(turn - rint(turn)), &sine, &cosine);
        turns[parity][r][0][f] = cosine * a.scaling;
        turns[parity][r][1][f] = sine * a.scaling;
      }
      lds_barrier();   // (a place is written again two times on, a barrier after everybody has read it)
    }
    for (uint32_t r = 0; r < a.each && i0 + r < rows; ++r) {
      const uint32_t i = i0 + r, after = r + 1 < a.each && i + 1 < rows ? i + 1 : i0 + step;
      const uint64_t row = (uint32_t)s.start + i;
      const int token = s.base + (int)i;
      float y[8];
      floats_of(next, y);
      if (after < rows) next = load(after);
      if (of_q || of_k) {
        if (a.norm) {
          float sum = 0.0f;
#pragma unroll
          for (int e = 0; e < 8; ++e) sum += y[e] * y[e];
          sum *= 1.0f / D;   // (in front of the lanes' sum: 256 squares of 2^60 are 2^128)
          sum = __uint_as_float(of_lanes<(int)kLanes>(__float_as_uint(sum), [](uint32_t u, uint32_t v) { return __float_as_uint(__uint_as_float(u) + __uint_as_float(v)); }));
          const float over = rsqrtf(sum + a.eps);
#pragma unroll
          for (int e = 0; e < 8; ++e) y[e] = y[e] * over * weight[e];
        }
        if (a.rotary) turn<D>(a, turns[parity][r], lane, half, y);
      }
      if (here >= heads) continue;
      if (of_q || (of_k && a.k_out)) {
        int none;
        uint8_t* const to = of_q ? a.q_out + row * a.q_out_stride : a.k_out + row * a.k_out_stride;
        const u32x4 words = quantised<SPLITZIP_BF16, D>(y, none);
        if constexpr (STREAM) st_stream(reinterpret_cast<u32x4*>(to + 2 * ((uint64_t)head * D + 8 * lane)), words);
        else *reinterpret_cast<u32x4*>(to + 2 * ((uint64_t)head * D + 8 * lane)) = words;
      }
      if (of_q || token < 0) continue;
      const uint32_t page = pages.page((uint32_t)token), place = pages.place((uint32_t)token);
      int byte = 0;
      Lane8<KIND> words = quantised<KIND, D>(y, byte);
      if constexpr (KIND == SPLITZIP_BF16) {   // V as it came: rounding makes signalling NaN quiet
#pragma unroll
        for (int e = 0; e < 4; ++e) words[e] = of_k ? words[e] : byte_perm(__float_as_uint(y[2 * e + 1]), __float_as_uint(y[2 * e]), 0x07060302u);
      }
      const uint64_t at = token_offset(a.cache, page, place) + head * a.cache.head_stride + lane * kBits<KIND>;
      *reinterpret_cast<Lane8<KIND>*>((of_k ? a.cache.k : a.cache.v) + at) = words;
      if constexpr (KIND != SPLITZIP_BF16) {
        if (has_scale<KIND, D>(lane)) (of_k ? a.cache.k_scales : a.cache.v_scales)[scale_offset(a.cache, page, place, scale_row<KIND, D>(head, lane))] = (uint8_t)byte;
      }
    }
  }
}

#endif  // SPLITZIP_APPEND_HPP
