// SplitZip for MI355X: pages of a pool handed out and taken back by what the requests of a step ask for.  Part of the single translation unit
// cache.hip (included inside its anonymous namespace, behind cache.hpp).
//
// Sequence s keeps kept = min(keep_s, len_s) of its tokens and gets rows_s more: n = kept + rows_s, of need = ceil(n / P) pages, where it
// has held = ceil(len_s / P).  Pages [need, held) of its table's row go back, pages [held, need) are filled in.  The free pages are a
// stack F_0 .. F_(f-1); with g pages given back and t taken, both counted over the sequences in order,
//   the r-th page given back becomes F_(f + g - 1 - r), and then the r-th page taken is F_(f + g - 1 - r),  f := f + g - t:
// what a step took is put back by one that gives up just that, in the order in which it lay there.  starts are the prefix sums of rows; row i of the call,
// of sequence s, is token kept_s + i - starts_s, and its slot that token's page times P and the place in it.
//
// Nothing here is much work: lengths, counts and page numbers, 32 bits each, and 16 bytes a row.  It is bound by latency, of the sums over
// the sequences, which all else waits for.  One workgroup makes them, and what follows from them for lengths, starts, stack and tables; few rows are filled in by
// it as well, many by a second launch.
//
// Bound by latency.  48 sequences with up to 5 rows each: 4.6 us.  1000 sequences that give 16 000 pages back, or take them: 11.9 us with eight pages at a time per
// thread (four 12.2, sixteen 11.8; one at a time, and sums without DPP, 19.1); the entries of 250 000 rows 6.2 us (9.4 with every row's sequence looked for among all).
#ifndef SPLITZIP_ALLOT_HPP
#define SPLITZIP_ALLOT_HPP

constexpr uint32_t kAllotThreads = 1024, kAllotWaves = kAllotThreads / 64;
constexpr uint32_t kRowsHere = 4096;     // rows that the first launch fills in itself
constexpr uint32_t kFillRows = 1024;     // rows of a workgroup of the second
constexpr uint32_t kPages = 8;           // pages that a thread moves at a time

struct AllotArgs {
  uint32_t* table;
  int32_t *starts, *lens;
  const int32_t *rows, *keep;            // keep: or null
  uint32_t* stack;
  int32_t* state;                        // a splitzip_pool_state
  int64_t* slots;                        // [n_rows] or null, as the next two
  int32_t *row_seqs, *positions;
  uint32_t table_stride, n_seqs, capacity, n_pages, n_rows;
  uint32_t page_shift;
  uint32_t fill;                         // rows are filled in by the first launch
};

// what a sequence asks for
struct Wanted {
  uint32_t rows, kept, held, need;
  int64_t len;
  __device__ Wanted() : rows(0), kept(0), held(0), need(0), len(0) {}
  __device__ Wanted(const AllotArgs& a, uint32_t s) {
    const uint32_t old = (uint32_t)min(max(a.lens[s], 0), (int)a.capacity), pages = (1u << a.page_shift) - 1;
    rows = (uint32_t)max(a.rows[s], 0);
    kept = a.keep ? min((uint32_t)max(a.keep[s], 0), old) : old;
    len = (int64_t)kept + rows;
    held = (old + pages) >> a.page_shift;
    need = (uint32_t)((len + pages) >> a.page_shift);
  }
  __device__ uint32_t gives() const { return held > need ? held - need : 0; }
  __device__ uint32_t takes() const { return need > held ? need - held : 0; }
};

// of 64 numbers below 2^38 each (sums of up to 64 of 32 bits), the sum; their halves' sums stay in 32 bits
__device__ inline uint64_t wave_sum(uint64_t x) {
  return wave_last(wave_incl_scan((uint32_t)x & 0xffffu)) + ((uint64_t)wave_last(wave_incl_scan((uint32_t)(x >> 16))) << 16);
}
__device__ inline uint32_t wave_max(uint32_t v) {   // as wave_incl_scan
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x111, 0xf, 0xf, false));
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x112, 0xf, 0xf, false));
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x114, 0xf, 0xf, false));
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x118, 0xf, 0xf, false));
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x142, 0xa, 0xf, false));
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x143, 0xc, 0xf, false));
  return wave_last(v);
}

// the last of entries [0, n] of ascending starts (starts[0] = 0) that is not above i, i below starts[n]: the sequence that has row i
template <typename P>
__device__ inline uint32_t owner_of(const P starts, uint32_t n, uint32_t i) {
  uint32_t low = 0, high = n;   // starts[low] <= i < starts[high]
  while (high - low > 1) {
    const uint32_t mid = (low + high) / 2;
    if ((uint32_t)starts[mid] <= i) low = mid;
    else high = mid;
  }
  return low;
}
// row i of the call, of sequence s, whose rows start at `start`, `end` being the next one's
__device__ inline void fill_row(const AllotArgs& a, uint32_t i, uint32_t s, uint32_t start, uint32_t end) {
  const uint32_t t = (uint32_t)a.lens[s] - (end - start) + (i - start);
  if (a.slots) {
    const uint32_t page = a.table[(uint64_t)s * a.table_stride + (t >> a.page_shift)];
    a.slots[i] = (int64_t)(((uint64_t)page << a.page_shift) + (t & ((1u << a.page_shift) - 1)));
  }
  if (a.row_seqs) a.row_seqs[i] = (int32_t)s;
  if (a.positions) a.positions[i] = (int32_t)t;
}
__device__ inline void no_row(const AllotArgs& a, uint32_t i) {
  if (a.slots) a.slots[i] = -1;
  if (a.row_seqs) a.row_seqs[i] = -1;
  if (a.positions) a.positions[i] = -1;
}

__global__ void __launch_bounds__(kAllotThreads) cache_allot_kernel(AllotArgs a) {
  __shared__ uint64_t sum_rows[kAllotWaves], sum_gives[kAllotWaves], sum_takes[kAllotWaves];
  __shared__ uint32_t most_rows[kAllotWaves], most_len[kAllotWaves];
  __shared__ uint32_t scan_rows[kAllotWaves], scan_pages[kAllotWaves];
  __shared__ uint32_t moved[kAllotThreads + 1], column[kAllotThreads];   // of a chunk of sequences: pages moved before each, and the first's column
  __shared__ uint32_t here[kAllotThreads + 1];                          // starts, if they are no more than that
  const uint32_t lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const int32_t free_now = a.state[0];

  // the sums, which say whether the step can be taken
  uint64_t rows = 0, gives = 0, takes = 0;
  uint32_t high_rows = 0, high_len = 0;
  Wanted mine;   // of the first chunk, the only one as a rule
  for (uint32_t s = threadIdx.x; s < a.n_seqs; s += kAllotThreads) {
    const Wanted w(a, s);
    if (s == threadIdx.x) mine = w;
    rows += w.rows;
    gives += w.gives();
    takes += w.takes();
    high_rows = max(high_rows, w.rows);
    high_len = max(high_len, (uint32_t)w.len);   // below 2^32
  }
  rows = wave_sum(rows);
  gives = wave_sum(gives);
  takes = wave_sum(takes);
  high_rows = wave_max(high_rows);
  high_len = wave_max(high_len);
  if (lane == 0) {
    sum_rows[wave] = rows;
    sum_gives[wave] = gives;
    sum_takes[wave] = takes;
    most_rows[wave] = high_rows;
    most_len[wave] = high_len;
  }
  __syncthreads();
  rows = gives = takes = 0;
  for (uint32_t w = 0; w < kAllotWaves; ++w) {
    rows += sum_rows[w];
    gives += sum_gives[w];
    takes += sum_takes[w];
    high_rows = max(high_rows, most_rows[w]);
    high_len = max(high_len, most_len[w]);
  }
  uint32_t status = 0;
  if (high_len > a.capacity) status |= SPLITZIP_ALLOT_LENGTH;
  if (rows > a.n_rows) status |= SPLITZIP_ALLOT_ROWS;
  if (free_now < 0 || (uint64_t)(uint32_t)free_now + gives > a.n_pages) status |= SPLITZIP_ALLOT_POOL;
  const uint64_t have = (uint64_t)(uint32_t)max(free_now, 0) + gives;
  if (!(status & SPLITZIP_ALLOT_POOL) && takes > have) status |= SPLITZIP_ALLOT_PAGES;
  if (threadIdx.x == 0) {
    int32_t* const st = a.state;
    st[1] = (int32_t)status;
    st[2] = status & SPLITZIP_ALLOT_PAGES ? (int32_t)min(takes - have, (uint64_t)0x7fffffff) : 0;
    if (!status) st[0] = (int32_t)(have - takes);
    st[3] = status ? 0 : (int32_t)rows;
    st[4] = status ? 0 : (int32_t)high_rows;
    st[5] = status ? 0 : (int32_t)high_len;
    st[6] = status ? 0 : (int32_t)takes;
    st[7] = status ? 0 : (int32_t)gives;
  }
  if (status) {   // nothing changes but the starts: a step without rows
    for (uint32_t s = threadIdx.x; s <= a.n_seqs; s += kAllotThreads) a.starts[s] = 0;
    if (a.fill)
      for (uint32_t i = threadIdx.x; i < a.n_rows; i += kAllotThreads) no_row(a, i);
    return;
  }

  // Pages, 1024 sequences at a time: first all that are given back, then, from the top, all that are taken.  Lengths change behind the last question
  // for them: with the first chunk kept in registers, in the last round.
  const uint32_t top = (uint32_t)have;
  for (int round = gives ? 0 : 1; round < 2; ++round) {
    uint32_t before_rows = 0, before_pages = 0;
    for (uint32_t s0 = 0; s0 < a.n_seqs; s0 += kAllotThreads) {
      const uint32_t s = s0 + threadIdx.x;
      Wanted w = mine;
      if (s0) w = s < a.n_seqs ? Wanted(a, s) : Wanted();
      const uint32_t pages = round ? w.takes() : w.gives();
      const uint32_t upto_rows = wave_incl_scan(w.rows), upto_pages = wave_incl_scan(pages);
      __syncthreads();   // (the chunk before this one has been read)
      if (lane == 63) {
        scan_rows[wave] = upto_rows;
        scan_pages[wave] = upto_pages;
      }
      __syncthreads();
      uint32_t wave_rows = 0, wave_pages = 0, all_rows = 0, all_pages = 0;
      for (uint32_t k = 0; k < kAllotWaves; ++k) {
        if (k < wave) {
          wave_rows += scan_rows[k];
          wave_pages += scan_pages[k];
        }
        all_rows += scan_rows[k];
        all_pages += scan_pages[k];
      }
      const uint32_t end = before_rows + wave_rows + upto_rows;
      moved[threadIdx.x + 1] = wave_pages + upto_pages;
      column[threadIdx.x] = round ? w.held : w.need;
      if (round) {
        here[threadIdx.x + 1] = end;
        if (s < a.n_seqs) {
          a.starts[s + 1] = (int32_t)end;
          a.lens[s] = (int32_t)w.len;
        }
      }
      if (threadIdx.x == 0) {
        moved[0] = 0;
        if (!s0) {
          here[0] = 0;
          if (round) a.starts[0] = 0;
        }
      }
      __syncthreads();
      // several pages of a thread at a time, since each goes through what a search and a load take
      const auto move = [&](auto pages_at_a_time, uint32_t p0) {
        constexpr uint32_t N = decltype(pages_at_a_time)::value;
        // (the last one once more where there are no more: the same word to the same place)
        uint32_t p[N], low[N], page[N];
        uint32_t *entry[N], *place[N];
#pragma unroll
        for (uint32_t k = 0; k < N; ++k) {
          p[k] = min(p0 + k * kAllotThreads, all_pages - 1);
          low[k] = 0;
        }
#pragma unroll 1
        for (uint32_t step = kAllotThreads / 2; step > 0; step /= 2) {   // the last sequence that no more than p pages are moved before
#pragma unroll
          for (uint32_t k = 0; k < N; ++k) low[k] += moved[low[k] + step] <= p[k] ? step : 0;
        }
#pragma unroll
        for (uint32_t k = 0; k < N; ++k) {
          entry[k] = a.table + (uint64_t)(s0 + low[k]) * a.table_stride + column[low[k]] + (p[k] - moved[low[k]]);
          place[k] = a.stack + (top - 1 - (before_pages + p[k]));
          page[k] = round ? *place[k] : *entry[k];
        }
#pragma unroll
        for (uint32_t k = 0; k < N; ++k) *(round ? entry[k] : place[k]) = page[k];
      };
      uint32_t p0 = threadIdx.x;
      if (all_pages > kAllotThreads)
        for (; p0 < all_pages; p0 += kPages * kAllotThreads) move(std::integral_constant<uint32_t, kPages>(), p0);
      else if (p0 < all_pages) move(std::integral_constant<uint32_t, 1>(), p0);
      before_rows += all_rows;
      before_pages += all_pages;
    }
    __syncthreads();
  }
  if (!a.fill) return;
  const uint32_t n_rows = (uint32_t)rows;
  for (uint32_t i = threadIdx.x; i < a.n_rows; i += kAllotThreads) {
    if (i >= n_rows) {
      no_row(a, i);
    } else if (a.n_seqs <= kAllotThreads) {
      const uint32_t s = owner_of(here, a.n_seqs, i);
      fill_row(a, i, s, here[s], here[s + 1]);
    } else {
      const uint32_t s = owner_of(a.starts, a.n_seqs, i);
      fill_row(a, i, s, (uint32_t)a.starts[s], (uint32_t)a.starts[s + 1]);
    }
  }
}

// the same by all lanes of a wave for one row: 64 entries are looked at at a time
__device__ inline uint32_t owner_by_wave(const int32_t* starts, uint32_t n, uint32_t i, uint32_t lane) {
  uint32_t low = 0, high = n;
  while (high - low > 1) {
    const uint32_t step = (high - low + 63) / 64, at = low + lane * step;
    const uint32_t upto = (uint32_t)__popcll(__ballot(at < high && (uint32_t)starts[min(at, high - 1)] <= i));   // the first `upto` lanes, the first at least
    low += (upto - 1) * step;
    high = min(high, low + step);
  }
  return low;
}

// Many rows: 1024 of them per workgroup, which looks their sequences' starts up first.
__global__ void __launch_bounds__(kThreads) cache_allot_fill_kernel(AllotArgs a) {
  __shared__ uint32_t part[kFillRows + 1];
  const uint32_t lane = threadIdx.x % 64, first = blockIdx.x * kFillRows, n_rows = (uint32_t)a.starts[a.n_seqs];
  uint32_t low = 0, n = 0;
  if (first < n_rows) {
    low = owner_by_wave(a.starts, a.n_seqs, first, lane);
    n = owner_by_wave(a.starts, a.n_seqs, min(first + kFillRows, n_rows) - 1, lane) + 1 - low;
    // (sequences without rows may be more than that)
    if (n <= kFillRows)
      for (uint32_t k = threadIdx.x; k <= n; k += kThreads) part[k] = (uint32_t)a.starts[low + k];
  }
  __syncthreads();
#pragma unroll
  for (uint32_t k = 0; k < kFillRows; k += kThreads) {
    const uint32_t i = first + k + threadIdx.x;
    if (i >= a.n_rows) continue;
    if (i >= n_rows) {
      no_row(a, i);
    } else if (n <= kFillRows) {
      const uint32_t s = owner_of(part, n, i);
      fill_row(a, i, low + s, part[s], part[s + 1]);
    } else {
      const uint32_t s = low + owner_of(a.starts + low, n, i);
      fill_row(a, i, s, (uint32_t)a.starts[s], (uint32_t)a.starts[s + 1]);
    }
  }
}

#endif  // SPLITZIP_ALLOT_HPP
