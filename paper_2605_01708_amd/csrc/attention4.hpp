// SplitZip for MI355X: attention of few rows over a cache of 4-bit words.  Part of the single translation unit cache.hip (included
// inside its anonymous namespace, behind attention.hpp, whose formulas, products and shares these are).
//
// A head's row of 128 4-bit words is 64 bytes, half of a cache line.  Read by a wave of its own, as attention_tokens_kernel does, every line is asked
// for twice and in halves: reading alone, shuffled pages of 16 tokens and 8 heads of 128, 3.9 TB/s that way, 6.4 in whole lines.  So a workgroup takes as
// many heads as make up a line (4 of 64 elements, 2 of 128, 1 of 256), its four waves bring whole lines of a stage's tokens into LDS, a quarter
// each, and then work on a head and a part of the tokens each.  A stage is written into one half of LDS while the other is
// worked on: one barrier a stage.
//
// Bound by memory and, behind it, by instructions: 64 sequences of 501 to 12000 tokens, 8 heads of 128, 437 MB in 84 us (5.2 TB/s); the same
// work on the first stage's tokens alone, without further loads, 67.  131072 tokens of 4 heads: 20.7 us, 18.5 without further loads.  Three
// waves per SIMD: with the join 87.2 us for the 64 sequences, two 90.8, four, with 36 registers in memory, 132.  Weights in two parts, as over
// other words (attention.hpp); rounded to BF16 those 64 sequences take 86.3 us and 131072 tokens 27.5 for 28.5, and the result is 0.0021 of
// itself off in place of its own rounding's 0.0016.  One head of 128, two of 64: 4 and 2 registers in memory (6 and none with caps or slopes).
#ifndef SPLITZIP_ATTENTION4_HPP
#define SPLITZIP_ATTENTION4_HPP

// D: elements of a head, H: heads of the workgroup
template <int D, int H>
struct Stage4 {
  static constexpr int KS = D / 32, DV = D / 16;
  static constexpr int kRow = D / 2;                                  // bytes of a token and head
  static constexpr int kAll = H * kRow;                               // of a token, the workgroup's heads side by side
  static constexpr int kTw = kWaves / H;                              // waves of a head
  static constexpr int kSteps = kTw * 32 * kAll < 8192 && D == 64 && H > 1 ? 2 : 1;   // of 32 tokens, of a wave in a stage
  static constexpr int kTokens = 32 * kTw * kSteps;
  static constexpr int kHalf = kTokens * kAll;                        // bytes of K, or V, of a stage
  static constexpr int kUnits = kAll / 16;                            // 16-byte units of a token
  static constexpr int kLoads = kHalf / 1024 / kWaves;                // of K, or V, by a wave
  static constexpr int kGroupsOf = D / kGroup4;
  static constexpr int kScales = H * kGroupsOf * kTokens;             // bytes of scales of K, or V: [head][group][token]
  static constexpr int kScaleLoads = (2 * kScales + 1023) / 1024;     // of 256 bytes, by a wave
  static constexpr int kBytes = 2 * kHalf + 2 * kScales;
  static constexpr int KB = kRow / 4 < 16 ? kRow / 4 : 16;            // bytes of a row of K that a lane takes at a time, and how often
  static constexpr int KW = kRow / 4 / KB;
  static constexpr int VB = kRow / 16;                                // bytes of a token of V per lane
  static constexpr int VW = (VB + 3) / 4;
  typedef typename std::conditional<KB == 16, u32x4, u32x2>::type KPart;
  static_assert(kHalf % (1024 * kWaves) == 0 && kLoads >= 1, "every wave brings a part of a stage");

  // Where token `token` (of the stage) and unit `unit` of it lie, in units; both maps are their own inverses, and stay inside eight tokens.
  // K: the 16 rows of an operand (tokens 8 a + 4 b + c, a and c from 0 to 3) lie in 16 different units of the banks.
  __device__ static uint32_t k_row(uint32_t token) { return kUnits == 2 ? token ^ (token / 8 & 1) * 4 : token; }
  __device__ static uint32_t k_unit(uint32_t token, uint32_t unit) {
    const uint32_t mi = token / 8 % 4 * 4 + token % 4;
    return unit ^ (kUnits >= 16 ? mi : mi / (16 / kUnits));
  }
  // V: rows of four tokens, one of each eight, are read at a time
  __device__ static uint32_t v_row(uint32_t token) { return kUnits == 8 ? token ^ (token / 8 & 1) : token ^ (token / 8 & 3); }
  __device__ static uint32_t v_unit(uint32_t token, uint32_t unit) { return kUnits == 8 && H > 1 ? unit ^ (token / 16 & 1) * 4 : unit; }

  static constexpr int kTurns = kUnits == 8 ? 2 : 4;
  // 4 bytes per lane straight into LDS
  __device__ static void load4_to_lds(const uint8_t* from, uint8_t* to) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from, (__attribute__((address_space(3))) void*)to, 4, 0, 0);
  }

  // A wave's part of the stage from token t0 on.  pages: lane l has the page of token 4 l.
  __device__ static void ask(const Cache& c, const Pages& at_pages, const uint8_t* k_base, const uint8_t* v_base, const uint8_t* ks_base, const uint8_t* vs_base,
                             uint32_t pages, int t0, uint32_t last8, uint8_t* lds, uint32_t wave, uint32_t lane) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const uint32_t load = wave * kLoads + i, unit = load * 64 + lane, row = unit / kUnits, at = unit % kUnits;   // where the lane's 16 bytes come to lie
      uint32_t eight, page;
      if constexpr (kUnits == 8) {   // 1024 bytes are eight tokens
        eight = load;
        page = (uint32_t)__builtin_amdgcn_readlane((int)pages, (int)(2 * load));
      } else {
        eight = row / 8;
        page = (uint32_t)__shfl((int)pages, (int)(2 * eight));
      }
      const uint64_t from = token_offset(c, page, at_pages.place(min((uint32_t)t0 + 8 * eight, last8)));
      const uint32_t k_token = k_row(row), v_token = v_row(row), k_at = k_unit(k_token, at), v_at = v_unit(v_token, at);
      // (heads need not lie side by side)
      const uint64_t k_head = kUnits > kRow / 16 ? k_at / (kRow / 16) * c.head_stride : 0, v_head = kUnits > kRow / 16 ? v_at / (kRow / 16) * c.head_stride : 0;
      load_to_lds(k_base + from + (k_head + k_token % 8 * c.token_stride + k_at % (kRow / 16) * 16), lds + load * 1024);
      load_to_lds(v_base + from + (v_head + v_token % 8 * c.token_stride + v_at % (kRow / 16) * 16), lds + kHalf + load * 1024);
    }
#pragma unroll
    for (int i = 0; i < kScaleLoads; ++i) {
      const uint32_t load = wave * kScaleLoads + i, byte = load * 256 + lane * 4;
      if (load * 256 >= 2 * kScales) break;   // (the same for the wave)
      const bool of_v = load * 256 >= kScales;
      const uint32_t row = (byte - (of_v ? kScales : 0)) / kTokens, token = byte % kTokens;
      const uint64_t from = (uint64_t)(uint32_t)__shfl((int)pages, (int)(token / 4 & ~1u)) * c.scale_page_stride + (uint64_t)row * c.page_tokens +
                            at_pages.place(min((uint32_t)t0 + (token & ~7u), last8)) + token % 8;
      load4_to_lds((of_v ? vs_base : ks_base) + from, lds + 2 * kHalf + load * 256);
    }
  }
};

template <int D, int H, bool PLAIN>
__global__ void __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(D == 256 ? 2 : 3))) attention_tokens4_kernel(AttentionArgs args) {
  constexpr int KIND = SPLITZIP_FP4_E2M1;
  using S = Stage4<D, H>;
  constexpr int KS = S::KS, DV = S::DV, KW = S::KW, VW = S::VW, kTokens = S::kTokens;
  constexpr int kAtATime = D == 256 ? 2 : DV;   // elements of V that are made ready for the product (all 16 of 256: 12 registers spilled)
  constexpr int kRoom = 2 * S::kBytes > 4 * 64 * D ? 2 * S::kBytes : 4 * 64 * D;
  __shared__ __attribute__((aligned(1024))) uint8_t lds[kRoom];
  __shared__ float lds_stat[kWaves][16][2];
  const uint32_t lane = threadIdx.x % 64, wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / 64)), m = lane % 16, g = lane / 16;
  Share w;
  if (!w.start(lane)) return;
  const Cache c = args.cache;
  const float scale = PLAIN ? args.scale * kLog2e : 1.0f;
  const uint8_t *const k_base = c.k + w.head * c.head_stride, *const v_base = c.v + w.head * c.head_stride;
  const uint8_t *const ks_base = c.k_scales + (uint64_t)w.head * S::kGroupsOf * c.page_tokens, *const vs_base = c.v_scales + (uint64_t)w.head * S::kGroupsOf * c.page_tokens;
  const uint32_t head = wave % H, turn = wave / H;
  w.head += head;

  do {
    if (!w.first_rows()) continue;
    do {
      const uint32_t last8 = (uint32_t)(w.s.len - 1) & ~7u;   // tokens behind the sequence's end are read at its last eight
      const Pages at_pages(c, args.seqs, w.seq);
      uint32_t pages = 0;
      const auto ask_pages = [&](int t0) { pages = at_pages.entry(min((uint32_t)t0 + (4 * lane % kTokens & ~7u), last8)); };
      const auto ask = [&](int t0, int buf) {
        pages = at_pages.clamped(pages);
        S::ask(c, at_pages, k_base, v_base, ks_base, vs_base, pages, t0, last8, lds + buf * S::kBytes, wave, lane);
      };
      if (w.begin < w.end) {
        ask_pages(w.begin);
        ask(w.begin, 0);
        if (w.begin + kTokens < w.end) ask_pages(w.begin + kTokens);
      }
      Rows<KIND, D, 1> r;
      r.load(w, w.tile * 16, m, g);
      Bias<1> bias;
      if constexpr (!PLAIN) bias.load(w, r.row, w.tile * 16, m);
      State<D, 1> st;
      st.clear();
      bool odd = false;   // words of V were left out
      int buf = 0;
#pragma unroll 1
      for (int t0 = w.begin; t0 < w.end; t0 += kTokens, buf ^= 1) {
        memory_arrived();
        lds_barrier();   // everybody's part is there, and nobody reads the other half any more
        typename S::KPart k[S::kSteps][2][KW];
        uint32_t v[S::kSteps][8][VW];
        u32x2 ks[S::kSteps][KW], vs[S::kSteps];
        const uint8_t* const from = lds + buf * S::kBytes;
#pragma unroll
        for (int u = 0; u < S::kSteps; ++u) {
          const uint32_t t = 32 * (turn * S::kSteps + u);
#pragma unroll
          for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int i = 0; i < KW; ++i) {
              const uint32_t token = t + 8 * (m / 4) + 4 * b + m % 4, unit = head * (S::kRow / 16) + (S::KB == 16 ? 4 * i + g : g / 2);
              k[u][b][i] = *reinterpret_cast<const typename S::KPart*>(from + S::k_row(token) * S::kAll + S::k_unit(token, unit) * 16 + (S::KB == 16 ? 0 : g % 2 * 8));
            }
#pragma unroll
          for (int i = 0; i < KW; ++i)
            ks[u][i] = *reinterpret_cast<const u32x2*>(from + 2 * S::kHalf + (head * S::kGroupsOf + (S::KB == 16 ? 4 * i + g : g / 2)) * kTokens + t + 8 * (m / 4));
          const uint32_t byte = head * S::kRow + S::VB * m, eight = t + 8 * g;
          const uint8_t* const vat = from + S::kHalf + eight * S::kAll + S::v_unit(eight, byte / 16) * 16 + byte % 16;
          uint32_t shift[S::kTurns];   // of a row of the eight from its own place
#pragma unroll
          for (int e = 0; e < S::kTurns; ++e) shift[e] = S::v_row(eight + e) % 8 * S::kAll - e * S::kAll;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const uint8_t* const at = vat + (int)shift[e % S::kTurns] + e * S::kAll;
            if constexpr (S::VB < 4) v[u][e][0] = *reinterpret_cast<const uint16_t*>(at);
            else __builtin_memcpy(v[u][e], __builtin_assume_aligned(at, S::VB), S::VB);
          }
          vs[u] = *reinterpret_cast<const u32x2*>(from + 2 * S::kHalf + S::kScales + (head * S::kGroupsOf + m * DV / kGroup4) * kTokens + t + 8 * g);
        }
        lds_read();
        if (t0 + kTokens < w.end) {
          ask(t0 + kTokens, buf ^ 1);
          if (t0 + 2 * kTokens < w.end) ask_pages(t0 + 2 * kTokens);
        }
#pragma unroll
        for (int u = 0; u < S::kSteps; ++u) {
          const int tu = t0 + 32 * (int)(turn * S::kSteps + u);
          if (tu >= w.end) break;
          f32x4 x[1][2];
#pragma unroll
          for (int b = 0; b < 2; ++b) {
            x[0][b] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int t = 0; t < KS; ++t) {
              constexpr int kEach = S::KB / 4;   // steps of a part
              x[0][b] = mfma(as_bf16(from_fp4(k[u][b][t / kEach][t % kEach], ks[u][t / kEach][b] >> (8 * (m % 4)) & 0xffu)), r.q[0][t], x[0][b]);
            }
          }
          const bool all = r.see_all(w, tu, (int)kStep);
          const int t8 = tu + (int)(8 * g);
          if constexpr (!PLAIN) st.shape(w, bias, x, t8);
          if (__builtin_expect(!all, 0)) st.mask(w, r, x, t8);
          st.raise({st.highest(x[0]) * scale});
          bf16x8 p[2][1];
          st.weigh(scale, x, p);
          uint32_t byte[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) byte[e] = vs[u][e / 4] >> (8 * (e % 4)) & 0xffu;
#pragma unroll
          for (int j0 = 0; j0 < DV; j0 += kAtATime) {
            u32x4 vt[kAtATime];   // elements of the eight tokens
#pragma unroll
            for (int i = 0; i < 4; ++i) {
#pragma unroll
              for (int j = 0; j < kAtATime; j += 2) {
                const int at = j0 + j;
                const uint32_t w0 = fp4_pair_to_bf16(v[u][2 * i][at / 8], byte[2 * i], at % 8 / 2), w1 = fp4_pair_to_bf16(v[u][2 * i + 1][at / 8], byte[2 * i + 1], at % 8 / 2);
                vt[j][i] = evens(w0, w1);
                vt[j + 1][i] = odds(w0, w1);
              }
            }
            if (__builtin_expect(!all, 0)) odd |= finite_only(vt, t8, w.s.len);
#pragma unroll
            for (int j = 0; j < kAtATime; ++j) st.add(j0 + j, as_bf16(vt[j]), p);
          }
        }
      }
      if (__builtin_expect(__ballot(odd) != 0, 0)) {
        const auto element = [&](int j, int i) { return DV * (4 * g + i) + j; };
        for (int t = w.begin + 32 * (int)(turn * S::kSteps); t < w.end; t += kTokens) st.add_odd(w, r, t, min(t + 32 * S::kSteps, w.end), (int)kStep, element);
      }
      lds_barrier();   // (nobody reads the last stage any more)
      finish_tokens<D>(w, st, lds, 64 * D, lds_stat, wave, lane, H);
    } while (w.more_rows());
  } while (w.next(lane));
}

#endif  // SPLITZIP_ATTENTION4_HPP
