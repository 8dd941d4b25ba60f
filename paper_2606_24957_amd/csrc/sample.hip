// sample.hip -- next tokens from logits with temperature, top-k, top-p and min-p, and drafted tokens accepted or
// rejected against the target's logits, from given random numbers.
//
// The kept set of a row is a prefix of its tokens in rank order (logit descending, index ascending): the k best, of
// those the fewest whose weights reach top_p of the sum, of those the ones whose weight is at least min_p of the
// largest.  It is described by the rank of its last token.  Three kernels:
//   chunks  every workgroup takes a piece of a row: its largest logit, the sum of its weights against that, and where
//           a filter needs it a histogram of counts and sums over quarter octaves of the weight
//   rows    one workgroup a row joins these, finds the quarter octave in which the kept set ends, and reads the row
//           again for the tokens that it has to rank: where all that may be kept are few, it holds them in LDS, ranks
//           them and draws; otherwise it ranks those of the last quarter octave by histograms of ever finer ranges
//   rest    (verification) what is left of the target's distribution after the first rejected draft, and the draw
// Weights are computed in 64-bit floating point and summed as integers, so results do not depend on the order of
// work; see sample.hpp.
#include "sample.hpp"

namespace dustin {

namespace {

constexpr int kChunkThreads = 256;
constexpr int kRowThreads = 1024;
constexpr int kRowWaves = kRowThreads / kWave;
constexpr int kFew = 1024;   // tokens ranked by comparing each with each
constexpr int kList = 4096;  // tokens of the last quarter octave held in LDS

// 2^d for -46 <= d <= 0, within a few units of 2^-53: 2^d = 2^n 2^f, |f| <= 1/2, and the Taylor series of e^(f ln 2)
// to the 12th power (the next term is below 2^-52).
__device__ __forceinline__ double exp2_f64(double d) {
  const double n = __builtin_rint(d), t = (d - n) * 0.693147180559945309417;
  double s = 1.0 / 479001600.0;
  s = __builtin_fma(s, t, 1.0 / 39916800.0);
  s = __builtin_fma(s, t, 1.0 / 3628800.0);
  s = __builtin_fma(s, t, 1.0 / 362880.0);
  s = __builtin_fma(s, t, 1.0 / 40320.0);
  s = __builtin_fma(s, t, 1.0 / 5040.0);
  s = __builtin_fma(s, t, 1.0 / 720.0);
  s = __builtin_fma(s, t, 1.0 / 120.0);
  s = __builtin_fma(s, t, 1.0 / 24.0);
  s = __builtin_fma(s, t, 1.0 / 6.0);
  s = __builtin_fma(s, t, 0.5);
  s = __builtin_fma(s, t, 1.0);
  s = __builtin_fma(s, t, 1.0);
  return s * __hiloint2double((1023 + (int)n) << 20, 0);
}

// A row's settings.
struct Settings {
  bool greedy;
  double scale;  // log2(e) / temperature
  int k;         // 0: all
  double p, m;   // p >= 1: all
  __device__ __forceinline__ Settings(const SampleArgs& a, int b) {
    const float t = a.temperature ? a.temperature[b] : a.s_temperature;
    greedy = !(t > 0.f);
    scale = greedy ? 1.0 : 1.44269504088896340736 / (double)t;
    k = a.top_k ? a.top_k[b] : a.s_top_k;
    if (k <= 0 || k >= a.vocab) k = 0;
    const float pp = a.top_p ? a.top_p[b] : a.s_top_p;
    p = pp < 1.f ? (pp > 0.f ? (double)pp : 0.0) : 1.0;
    const float mm = a.min_p ? a.min_p[b] : a.s_min_p;
    m = mm > 0.f ? (mm < 1.f ? (double)mm : 1.0) : 0.0;
  }
  __device__ __forceinline__ bool filters() const { return !greedy && (k > 0 || p < 1.0); }
};

// Weight of logit x in a row (or chunk) whose largest is top.
__device__ __forceinline__ double weight(float x, float top, double scale) {
  if (x == top) return top == -INFINITY ? 0.0 : 1.0;
  const double d = ((double)x - (double)top) * scale;
  if (!(d > -45.5)) return 0.0;
  const double w = exp2_f64(d);
  return w < 0x1p-45 ? 0.0 : w;
}
// ... as a multiple of 2^-44 (the mantissa bits of w 2^44 + 2^52).
__device__ __forceinline__ uint64_t units(double w) {
  return (uint64_t)__double_as_longlong(__builtin_fma(w, 0x1p44, 0x1p52)) & 0xfffffffffffffull;
}

__device__ __forceinline__ uint64_t rank_of(float x, int i) {
  return ((uint64_t)~order_key(x) << kSampleIdxBits) | (uint32_t)i;
}
__device__ __forceinline__ float logit_of_key(uint32_t key) {
  return __uint_as_float((key & 0x80000000u) ? key & 0x7fffffffu : ~key);
}
__device__ __forceinline__ float logit_of_rank(uint64_t r) { return logit_of_key(~(uint32_t)(r >> kSampleIdxBits)); }

// Quarter octave of a logit (an integer, ascending with it).
__device__ __forceinline__ double octave(float x, double scale) { return __builtin_floor((double)x * scale * 4.0); }

// A row in 16-byte pieces: piece g holds tokens first(g) .. first(g) + n - 1.  Logits that are NaN, and tokens outside
// the row, come as -infinity.
template <bool kBf16>
struct RowReader {
  static constexpr int n = kBf16 ? 8 : 4;
  const char* row;
  int skew, vocab;
  __device__ __forceinline__ RowReader(const SampleArgs& a, int b, int t) {
    const int64_t at = b * a.sb + t * a.st;
    row = static_cast<const char*>(a.logits) + at * (kBf16 ? 2 : 4);
    skew = (int)(((uintptr_t)row & 15) / (kBf16 ? 2 : 4));
    vocab = a.vocab;
  }
  __device__ __forceinline__ int first(int g) const { return g * n - skew; }
  __device__ __forceinline__ float at(int i) const {
    const float x = kBf16 ? bf16_bits_to_float(reinterpret_cast<const uint16_t*>(row)[i])
                          : reinterpret_cast<const float*>(row)[i];
    return x != x ? -INFINITY : x;
  }
  __device__ __forceinline__ void read(int g, float (&x)[n]) const {
    const int i0 = first(g);
    if (i0 >= 0 && i0 + n <= vocab) {
      const u32x4 v = *reinterpret_cast<const u32x4*>(row + (int64_t)i0 * (kBf16 ? 2 : 4));
#pragma unroll
      for (int e = 0; e < n; ++e) {
        if constexpr (kBf16) x[e] = __uint_as_float((e & 1) ? v[e / 2] & 0xffff0000u : v[e / 2] << 16);
        else x[e] = __uint_as_float(v[e]);
        if (x[e] != x[e]) x[e] = -INFINITY;
      }
    } else {
#pragma unroll
      for (int e = 0; e < n; ++e) x[e] = i0 + e >= 0 && i0 + e < vocab ? at(i0 + e) : -INFINITY;
    }
  }
};

__device__ __forceinline__ uint64_t shfl_xor_u64(uint64_t x, int d) {
  return (uint64_t)__shfl_xor((unsigned long long)x, d);
}
__device__ __forceinline__ uint64_t wave_min(uint64_t x) {
#pragma unroll
  for (int d = 1; d < kWave; d *= 2) {
    const uint64_t y = shfl_xor_u64(x, d);
    x = y < x ? y : x;
  }
  return x;
}
__device__ __forceinline__ uint64_t wave_sum(uint64_t x) {
#pragma unroll
  for (int d = 1; d < kWave; d *= 2) x += shfl_xor_u64(x, d);
  return x;
}
__device__ __forceinline__ uint64_t wave_scan(uint64_t x) {  // inclusive
  const int lane = threadIdx.x & (kWave - 1);
#pragma unroll
  for (int d = 1; d < kWave; d *= 2) {
    const uint64_t y = (uint64_t)__shfl_up((unsigned long long)x, d);
    if (lane >= d) x += y;
  }
  return x;
}

// Sum over a workgroup of `waves` waves, for every thread.
template <int waves>
__device__ __forceinline__ uint64_t block_sum(uint64_t x, uint64_t* sm) {
  x = wave_sum(x);
  __syncthreads();
  if ((threadIdx.x & (kWave - 1)) == 0) sm[threadIdx.x / kWave] = x;
  __syncthreads();
  uint64_t s = 0;
#pragma unroll
  for (int w = 0; w < waves; ++w) s += sm[w];
  return s;
}
// The sums of the threads before this one, and of all.
template <int waves>
__device__ __forceinline__ uint64_t block_before(uint64_t x, uint64_t* sm, uint64_t& all) {
  const uint64_t incl = wave_scan(x);
  __syncthreads();
  if ((threadIdx.x & (kWave - 1)) == kWave - 1) sm[threadIdx.x / kWave] = incl;
  __syncthreads();
  uint64_t base = 0;
  all = 0;
#pragma unroll
  for (int w = 0; w < waves; ++w) {
    base += w < (int)threadIdx.x / kWave ? sm[w] : 0;
    all += sm[w];
  }
  return base + incl - x;
}

template <bool kBf16>
__global__ __launch_bounds__(kChunkThreads) void sample_chunk_kernel(SampleArgs a) {
  constexpr int n = RowReader<kBf16>::n, kMost = kRowThreads / kChunkThreads;  // pieces of a thread, at most
  __shared__ unsigned long long sm_sum[kChunkThreads / kWave][kSampleBins];
  __shared__ uint32_t sm_cnt[kChunkThreads / kWave][kSampleBins];
  __shared__ uint64_t sm_red[kChunkThreads / kWave];
  const int chunk = blockIdx.x, r = blockIdx.y, wave = threadIdx.x / kWave;
  const int b = r / a.rows_per_seq, t = r - b * a.rows_per_seq;
  if (a.n_query && t >= a.n_query[b]) return;
  const RowReader<kBf16> row(a, b, t);
  const Settings s(a, b);
  float x[kMost][n];
  uint64_t best = ~0ull;
#pragma unroll
  for (int j = 0; j < kMost; ++j) {
    const int g = j * kChunkThreads + threadIdx.x;
#pragma unroll
    for (int e = 0; e < n; ++e) x[j][e] = -INFINITY;
    if (g < a.granules) row.read(chunk * a.granules + g, x[j]);
  }
#pragma unroll
  for (int j = 0; j < kMost; ++j)
#pragma unroll
    for (int e = 0; e < n; ++e) {
      const int i = row.first(chunk * a.granules + j * kChunkThreads + (int)threadIdx.x) + e;
      const uint64_t k = rank_of(x[j][e], i & (kSampleMaxVocab - 1));
      best = x[j][e] != -INFINITY && k < best ? k : best;
    }
  const bool filters = s.filters();
  if (filters)
    for (int i = threadIdx.x & (kWave - 1); i < kSampleBins; i += kWave) {
      sm_sum[wave][i] = 0;
      sm_cnt[wave][i] = 0;
    }
  best = wave_min(best);
  if ((threadIdx.x & (kWave - 1)) == 0) sm_red[wave] = best;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kChunkThreads / kWave; ++w) best = sm_red[w] < best ? sm_red[w] : best;
  const float top = best == ~0ull ? -INFINITY : logit_of_rank(best);
  uint64_t sum = 0;
  if (!s.greedy && best != ~0ull) {
    const double oct = octave(top, s.scale);
#pragma unroll
    for (int j = 0; j < kMost; ++j)
#pragma unroll
      for (int e = 0; e < n; ++e) {
        const uint64_t w = units(weight(x[j][e], top, s.scale));
        if (!w) continue;
        sum += w;
        if (filters) {
          const int bin = x[j][e] == top ? 0 : (int)(oct - octave(x[j][e], s.scale));
          atomicAdd(&sm_sum[wave][bin], (unsigned long long)w);
          atomicAdd(&sm_cnt[wave][bin], 1u);
        }
      }
  }
  sum = block_sum<kChunkThreads / kWave>(sum, sm_red);
  const int64_t at = (int64_t)r * a.chunks + chunk;
  if (threadIdx.x == 0) {
    a.c_top[at] = top;
    a.c_best[at] = best;
    a.c_sum[at] = sum;
  }
  if (filters && threadIdx.x < kSampleBins) {
    unsigned long long h = 0;
    uint32_t c = 0;
#pragma unroll
    for (int w = 0; w < kChunkThreads / kWave; ++w) {
      h += sm_sum[w][threadIdx.x];
      c += sm_cnt[w][threadIdx.x];
    }
    a.h_sum[at * kSampleBins + threadIdx.x] = h;
    a.h_cnt[at * kSampleBins + threadIdx.x] = c;
  }
}

// A chunk's sum of weights, in units of the row's.
__device__ __forceinline__ uint64_t rescaled(uint64_t sum, float c_top, float top, double scale) {
  if (c_top == top) return sum;
  const double d = ((double)c_top - (double)top) * scale;
  return d > -110.0 ? (uint64_t)((double)sum * (d > -46.0 ? exp2_f64(d) : exp2_f64(d + 64.0) * 0x1p-64)) : 0;
}

// Of the tokens of a chunk (one piece to a thread) with rank at most `last`, the one at which the running sum of
// `value` passes `target` (the last with any, if none does); -1 where no token has any.
template <bool kBf16, class Value>
__device__ int draw_in_chunk(const SampleArgs& a, const RowReader<kBf16>& row, int chunk, uint64_t target, Value value,
                             uint64_t* sm, int* sm_token) {
  constexpr int n = RowReader<kBf16>::n;
  uint64_t v[n], own = 0;
  int i0 = 0;
#pragma unroll
  for (int e = 0; e < n; ++e) v[e] = 0;
  if ((int)threadIdx.x < a.granules) {
    const int g = chunk * a.granules + threadIdx.x;
    float x[n];
    row.read(g, x);
    i0 = row.first(g);
#pragma unroll
    for (int e = 0; e < n; ++e) {
      v[e] = x[e] == -INFINITY ? 0 : value(x[e], i0 + e);
      own += v[e];
    }
  }
  if (threadIdx.x == 0) *sm_token = -1;
  uint64_t all;
  uint64_t run = block_before<kRowWaves>(own, sm, all);
  if (all && target >= all) target = all - 1;
#pragma unroll
  for (int e = 0; e < n; ++e) {
    if (run <= target && target < run + v[e]) *sm_token = i0 + e;
    run += v[e];
  }
  __syncthreads();
  return *sm_token;
}

// The chunk at which the running sum of value(c) passes floor(u * whole sum), and what is left of that target in it.
template <class Value>
__device__ int draw_chunk(const SampleArgs& a, float u, Value value, uint64_t* sm, int* sm_chunk, uint64_t* sm_rest,
                          uint64_t& all) {
  const uint64_t v = (int)threadIdx.x < a.chunks ? value((int)threadIdx.x) : 0;
  if (threadIdx.x == 0) *sm_chunk = -1;
  const uint64_t run = block_before<kRowWaves>(v, sm, all);
  u = u > 0.f ? u : 0.f;
  uint64_t target = (uint64_t)((double)u * (double)all);
  if (all && target >= all) target = all - 1;
  if (run <= target && target < run + v) {
    *sm_chunk = threadIdx.x;
    *sm_rest = target - run;
  }
  __syncthreads();
  return *sm_chunk;
}

template <bool kBf16, bool kDraw>
__global__ __launch_bounds__(kRowThreads) void sample_row_kernel(SampleArgs a) {
  constexpr int n = RowReader<kBf16>::n;
  __shared__ uint64_t sm_rank[kList];
  __shared__ uint64_t sm_w[kList];
  __shared__ unsigned long long sm_sum[1024];  // histogram: of quarter octaves, then of ranges of ranks
  __shared__ uint32_t sm_cnt[1024];
  __shared__ unsigned long long sm_chunk_sum[kSampleMaxChunks];
  __shared__ uint64_t sm_red[kRowWaves], sm_u64[4];
  __shared__ int sm_int[2];
  __shared__ uint32_t sm_n;
  const int r = blockIdx.x, tid = threadIdx.x;
  const int b = r / a.rows_per_seq, t = r - b * a.rows_per_seq;
  if (a.n_query && t >= a.n_query[b]) return;
  const RowReader<kBf16> row(a, b, t);
  const Settings s(a, b);
  const int64_t c0 = (int64_t)r * a.chunks;
  const int pieces = a.granules * a.chunks;

  // ---- the row's best token
  uint64_t best = tid < a.chunks ? a.c_best[c0 + tid] : ~0ull;
  best = wave_min(best);
  if ((tid & (kWave - 1)) == 0) sm_red[tid / kWave] = best;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kRowWaves; ++w) best = sm_red[w] < best ? sm_red[w] : best;
  if (best == ~0ull || s.greedy) {  // nothing to draw from, or nothing to draw
    if (tid == 0) {
      const bool none = best == ~0ull;
      a.row[r] = {none ? 0 : best, none ? 0 : 1ull << kSampleFrac, none ? -INFINITY : logit_of_rank(best)};
      if constexpr (kDraw) a.token[b] = none ? -1 : (int)(best & (kSampleMaxVocab - 1));
    }
    return;
  }
  const float top = logit_of_rank(best);
  auto units_of = [&](float x) { return units(weight(x, top, s.scale)); };
  // calls f(x, i) for every token of the row whose rank lies in [lo, hi]
  auto each = [&](uint64_t lo, uint64_t hi, auto f) {
    const uint32_t key_hi = ~(uint32_t)(lo >> kSampleIdxBits), key_lo = ~(uint32_t)(hi >> kSampleIdxBits);
    for (int g = tid; g < pieces; g += kRowThreads) {
      float x[n];
      row.read(g, x);
#pragma unroll
      for (int e = 0; e < n; ++e) {
        const uint32_t k = order_key(x[e]);
        if (x[e] != -INFINITY && k >= key_lo && k <= key_hi) {
          const uint64_t c = rank_of(x[e], row.first(g) + e);
          if (c >= lo && c <= hi) f(x[e], c);
        }
      }
    }
  };
  // least key whose logit satisfies a condition that holds from some logit on
  auto least_key = [&](auto holds) {
    uint32_t lo = 0, hi = order_key(top);  // holds(hi)
    while (lo < hi) {
      const uint32_t mid = lo + (hi - lo) / 2;
      if (holds(logit_of_key(mid))) hi = mid;
      else lo = mid + 1;
    }
    return lo;
  };
  auto whole_key = [](uint32_t key) { return ((uint64_t)~key << kSampleIdxBits) | (kSampleMaxVocab - 1); };

  uint64_t last = ~0ull;  // rank of the last kept token
  int last_bin = -1;      // its quarter octave, with a histogram
  if (s.filters()) {
    // ---- histogram of the row
    const double oct = octave(top, s.scale);
    for (int i = tid; i < 1024; i += kRowThreads) {
      sm_sum[i] = 0;
      sm_cnt[i] = 0;
    }
    if (tid == 0) sm_n = 0;
    __syncthreads();
    for (int e = tid; e < a.chunks * kSampleBins; e += kRowThreads) {
      const int c = e / kSampleBins, bin = e - c * kSampleBins;
      const uint32_t cnt = a.h_cnt[c0 * kSampleBins + e];
      const float c_top = a.c_top[c0 + c];
      const double off = c_top == top ? 0.0 : oct - octave(c_top, s.scale);
      if (cnt && off + bin < kSampleBins) {
        atomicAdd(&sm_cnt[(int)off + bin], cnt);
        atomicAdd(&sm_sum[(int)off + bin], (unsigned long long)rescaled(a.h_sum[c0 * kSampleBins + e], c_top, top, s.scale));
      }
    }
    __syncthreads();
    uint64_t all_cnt, all_sum;
    const uint64_t my_cnt = tid < kSampleBins ? sm_cnt[tid] : 0, my_sum = tid < kSampleBins ? sm_sum[tid] : 0;
    const uint64_t cnt_before = block_before<kRowWaves>(my_cnt, sm_red, all_cnt);
    const uint64_t sum_before = block_before<kRowWaves>(my_sum, sm_red, all_sum);
    // ends of quarter octaves: a token lies in bin j or a better one iff its key is at least bin_key(j)
    auto bin_key = [&](int j) { return least_key([&](float x) { return oct - octave(x, s.scale) <= j; }); };
    // the first bin whose running count (or sum) reaches a target; the counts and sums before it and in it
    struct Bin {
      int j;
      uint64_t cnt, sum, in;
    };
    auto find_bin = [&](bool by_sum, double target) {
      __syncthreads();
      if (tid == 0) sm_int[0] = kSampleBins - 1;
      __syncthreads();
      const double reach = by_sum ? (double)(sum_before + my_sum) : (double)(cnt_before + my_cnt);
      if (tid < kSampleBins && my_cnt && reach >= target) atomicMin(&sm_int[0], tid);
      __syncthreads();
      const int j = sm_int[0];
      if (tid == j) {
        sm_u64[0] = cnt_before;
        sm_u64[1] = sum_before;
        sm_u64[2] = my_cnt;
      }
      __syncthreads();
      return Bin{j, sm_u64[0], sm_u64[1], sm_u64[2]};
    };
    const bool by_count = s.k > 0 && (uint64_t)s.k < all_cnt;
    Bin bin = by_count ? find_bin(false, s.k) : find_bin(true, s.p * (double)all_sum);
    if (bin.cnt + bin.in <= kFew) {
      // ---- few: all that may be kept, in LDS, each compared with each
      each(0, whole_key(bin_key(bin.j)), [&](float x, uint64_t c) {
        const uint64_t w = units_of(x);
        if (!w) return;
        const uint32_t at = atomicAdd(&sm_n, 1u);
        if (at < kFew) {
          sm_rank[at] = c;
          sm_w[at] = w;
        }
      });
      __syncthreads();
      const int m = min((int)sm_n, kFew);
      int share = 64;  // threads to a token
      while (share * m > kRowThreads) share >>= 1;
      const int e = tid / share, part = tid % share;
      const bool mine = e < m;
      const uint64_t c = mine ? sm_rank[e] : 0, w = mine ? sm_w[e] : 0;
      uint64_t place = 0, before = 0;
      if (mine)
        for (int j = part; j < m; j += share)
          if (sm_rank[j] < c) {
            ++place;
            before += sm_w[j];
          }
      for (int d = 1; d < share; d *= 2) {
        place += shfl_xor_u64(place, d);
        before += shfl_xor_u64(before, d);
      }
      bool kept = mine && (s.k == 0 || place < (uint64_t)s.k);
      const uint64_t z_k = by_count ? block_sum<kRowWaves>(kept && part == 0 ? w : 0, sm_red) : all_sum;
      if (s.p < 1.0) kept &= place == 0 || (double)before < s.p * (double)z_k;
      kept &= place == 0 || weight(logit_of_rank(c), top, s.scale) >= s.m;
      const uint64_t z = block_sum<kRowWaves>(kept && part == 0 ? w : 0, sm_red);
      if (tid == 0) {
        sm_u64[3] = 0;
        sm_int[1] = -1;
      }
      __syncthreads();
      if (kept && part == 0) atomicMax(reinterpret_cast<unsigned long long*>(&sm_u64[3]), (unsigned long long)c);
      if (mine && part == 0) sm_w[e] = kept ? w : 0;
      __syncthreads();
      if constexpr (kDraw) {
        float u = a.u[b];
        u = u > 0.f ? u : 0.f;
        uint64_t target = (uint64_t)((double)u * (double)z);
        if (target >= z) target = z - 1;
        const uint32_t i = (uint32_t)c & (kSampleMaxVocab - 1);
        uint64_t run = 0;
        if (kept)
          for (int j = part; j < m; j += share)
            if (((uint32_t)sm_rank[j] & (kSampleMaxVocab - 1)) < i) run += sm_w[j];
        for (int d = 1; d < share; d *= 2) run += shfl_xor_u64(run, d);
        if (kept && part == 0 && run <= target && target < run + w) a.token[b] = (int)i;
      }
      if (tid == 0) a.row[r] = {sm_u64[3], z, top};
      return;
    }
    // ---- many: the last token by ever finer ranges of ranks
    uint64_t list_lo = 1, list_hi = 0;  // ranks whose tokens are in the list
    int list_n = 0;
    auto each_of = [&](uint64_t lo, uint64_t hi, auto f) {  // f(rank, units)
      if (list_lo <= lo && hi <= list_hi) {
        for (int j = tid; j < list_n; j += kRowThreads)
          if (sm_rank[j] >= lo && sm_rank[j] <= hi) f(sm_rank[j], sm_w[j]);
      } else {
        each(lo, hi, [&](float x, uint64_t c) {
          const uint64_t w = units_of(x);
          if (w) f(c, w);
        });
      }
    };
    // the first token, from bin `at` on, at which the running count (sum) reaches the target; sum up to it
    auto find_token = [&](const Bin& at, bool by_sum, double target, uint64_t& sum) {
      uint64_t lo = at.j == 0 ? 0 : whole_key(bin_key(at.j - 1)) + 1, hi = whole_key(bin_key(at.j));
      uint64_t cnt_b = at.cnt, sum_b = at.sum;
      if (!(list_lo <= lo && hi <= list_hi) && at.in <= kList) {
        __syncthreads();
        if (tid == 0) sm_n = 0;
        __syncthreads();
        each(lo, hi, [&](float x, uint64_t c) {
          const uint64_t w = units_of(x);
          if (!w) return;
          const uint32_t j = atomicAdd(&sm_n, 1u);
          if (j < kList) {
            sm_rank[j] = c;
            sm_w[j] = w;
          }
        });
        __syncthreads();
        list_n = min((int)sm_n, kList);
        list_lo = lo;
        list_hi = hi;
      }
      for (;;) {
        const int bits = 64 - __clzll((long long)(hi - lo));  // hi > lo, or 0
        const int shift = hi == lo ? 0 : bits > 10 ? bits - 10 : 0;
        __syncthreads();
        sm_sum[tid] = 0;
        sm_cnt[tid] = 0;
        if (tid == 0) sm_int[0] = 1 << 20;
        __syncthreads();
        each_of(lo, hi, [&](uint64_t c, uint64_t w) {
          const int j = (int)((c - lo) >> shift);
          atomicAdd(&sm_cnt[j], 1u);
          atomicAdd(&sm_sum[j], (unsigned long long)w);
        });
        __syncthreads();
        const uint64_t oc = sm_cnt[tid], os = sm_sum[tid];
        uint64_t x;
        const uint64_t cb = cnt_b + block_before<kRowWaves>(oc, sm_red, x);
        const uint64_t sb = sum_b + block_before<kRowWaves>(os, sm_red, x);
        if (oc && (by_sum ? (double)(sb + os) : (double)(cb + oc)) >= target) atomicMin(&sm_int[0], tid);
        __syncthreads();
        if (sm_int[0] == 1 << 20) {  // (sums of the histogram and of the tokens differ in the last place)
          __syncthreads();
          if (tid == 0) sm_int[0] = -1;
          __syncthreads();
          if (oc) atomicMax(&sm_int[0], tid);
          __syncthreads();
        }
        const int j = max(sm_int[0], 0);
        if (tid == j) {
          sm_u64[0] = cb;
          sm_u64[1] = sb;
          sm_u64[2] = sb + os;
        }
        __syncthreads();
        cnt_b = sm_u64[0];
        sum_b = sm_u64[1];
        sum = sm_u64[2];
        lo += (uint64_t)j << shift;
        if (shift == 0) return lo;
        const uint64_t end = lo + ((1ull << shift) - 1);
        hi = end < hi ? end : hi;
      }
    };
    uint64_t z_k = all_sum;
    last_bin = kSampleBins - 1;
    if (by_count) {
      last = find_token(bin, false, s.k, z_k);
      last_bin = bin.j;
    }
    if (s.p < 1.0) {
      if (by_count) {  // the histogram of ranges has taken the place of that of quarter octaves: both are in registers
        bin = find_bin(true, s.p * (double)z_k);
      }
      uint64_t x;
      const uint64_t at = find_token(bin, true, s.p * (double)z_k, x);
      if (at < last) {
        last = at;
        last_bin = bin.j;
      }
    }
  }
  if (s.m > 0.0) {
    const uint64_t at = whole_key(least_key([&](float x) { return weight(x, top, s.scale) >= s.m; }));
    if (at < last) {
      last = at;
      last_bin = s.filters() ? (int)(octave(top, s.scale) - octave(logit_of_rank(at), s.scale)) : -1;
    }
  }

  // ---- sums of the kept weights by chunks
  __syncthreads();
  if (tid < a.chunks) sm_chunk_sum[tid] = 0;
  __syncthreads();
  if (last == ~0ull) {
    if (tid < a.chunks) sm_chunk_sum[tid] = rescaled(a.c_sum[c0 + tid], a.c_top[c0 + tid], top, s.scale);
  } else {
    uint64_t from = 0;  // ranks that the histograms do not give
    if (last_bin >= 0) {
      const double oct = octave(top, s.scale);
      for (int e = tid; e < a.chunks * kSampleBins; e += kRowThreads) {
        const int c = e / kSampleBins, bin = e - c * kSampleBins;
        const uint64_t sum = a.h_sum[c0 * kSampleBins + e];
        const float c_top = a.c_top[c0 + c];
        const double off = c_top == top ? 0.0 : oct - octave(c_top, s.scale);
        if (sum && off + bin < last_bin)
          atomicAdd(&sm_chunk_sum[c], (unsigned long long)rescaled(sum, c_top, top, s.scale));
      }
      if (last_bin > 0) {
        const int j = last_bin - 1;
        from = whole_key(least_key([&](float x) { return oct - octave(x, s.scale) <= j; })) + 1;
      }
    }
    const uint32_t inv = a.granules * n;
    each(from, last, [&](float x, uint64_t c) {
      const uint64_t w = units_of(x);
      const uint32_t i = (uint32_t)c & (kSampleMaxVocab - 1);
      if (w) atomicAdd(&sm_chunk_sum[(i + row.skew) / inv], (unsigned long long)w);
    });
  }
  __syncthreads();
  uint64_t z;
  const int chunk = draw_chunk(a, kDraw ? a.u[b] : 0.f, [&](int c) { return (uint64_t)sm_chunk_sum[c]; }, sm_red,
                               &sm_int[0], &sm_u64[0], z);
  if (tid == 0) a.row[r] = {last, z, top};
  if constexpr (kDraw) {
    if (chunk < 0) return;
    const int token = draw_in_chunk<kBf16>(
        a, row, chunk, sm_u64[0], [&](float x, int i) { return rank_of(x, i) <= last ? units_of(x) : 0; }, sm_red,
        &sm_int[1]);
    if (tid == 0) a.token[b] = token;
  }
}

// The kept tokens' probabilities, 0 for the others.
template <bool kBf16>
__global__ __launch_bounds__(kChunkThreads) void sample_probs_kernel(SampleArgs a) {
  const int b = blockIdx.y;
  const int i = blockIdx.x * kChunkThreads + threadIdx.x;
  if (i >= a.vocab) return;
  const RowReader<kBf16> row(a, b, 0);
  const Settings s(a, b);
  const SampleRow o = a.row[b];
  const float x = row.at(i);
  double p = 0.0;
  if (o.sum && x != -INFINITY && rank_of(x, i) <= o.last)
    p = weight(x, o.top, s.scale) / ((double)o.sum * 0x1p-44);
  a.probs[b * a.probs_sb + i] = (float)p;
}

// A window's accepted drafts, and a chunk's share of the distribution that the next token is drawn from; the last
// workgroup of a sequence draws it.
template <bool kBf16>
__global__ __launch_bounds__(kRowThreads) void verify_rest_kernel(SampleArgs a) {
  constexpr int n = RowReader<kBf16>::n;
  __shared__ uint64_t sm_red[kRowWaves], sm_u64[2];
  __shared__ int sm_int[3];
  const int chunk = blockIdx.x, b = blockIdx.y, tid = threadIdx.x;
  const int T = a.n_query ? clampi(a.n_query[b], 0, a.rows_per_seq) : a.rows_per_seq;
  const Settings s(a, b);
  if (T == 0) {
    if (chunk == 0 && tid == 0) {
      a.accepted[b] = 0;
      a.token[b] = -1;
    }
    return;
  }
  // ---- accepted drafts: draft t where u q(x) < p(x), up to the first that is not
  if (tid < kWave) {
    bool ok = false;
    if (tid < T - 1) {
      const int x = a.draft[b * a.draft_sb + tid];
      const SampleRow o = a.row[b * a.rows_per_seq + tid];
      if (x >= 0 && x < a.vocab && o.sum) {
        const float l = RowReader<kBf16>(a, b, tid).at(x);
        const double p = l != -INFINITY && rank_of(l, x) <= o.last ? weight(l, o.top, s.scale) / ((double)o.sum * 0x1p-44) : 0.0;
        const double q = a.q ? (double)a.q[b * a.q_sb + tid * a.q_st + x] : 1.0;
        ok = (double)a.u_accept[b * a.ua_sb + tid] * q < p;
      }
    }
    const uint64_t no = ~__ballot(ok);
    if (tid == 0) sm_int[0] = min((int)__builtin_ctzll(no), T - 1);
  }
  __syncthreads();
  const int kept = sm_int[0];
  const bool rejected = kept < T - 1;
  const RowReader<kBf16> row(a, b, kept);
  const SampleRow o = a.row[b * a.rows_per_seq + kept];
  const int x_draft = rejected ? a.draft[b * a.draft_sb + kept] : -1;
  const float* q = rejected && a.q ? a.q + b * a.q_sb + kept * a.q_st : nullptr;
  const double z = (double)o.sum * 0x1p-44;
  // probabilities as multiples of 2^-60
  auto whole = [&](float x, int i) -> double {
    return rank_of(x, i) <= o.last ? weight(x, o.top, s.scale) / z : 0.0;
  };
  auto rest = [&](double p, int i) {
    if (rejected) p -= q ? (double)q[i] : i == x_draft ? 1.0 : 0.0;
    return p > 0.0 ? p : 0.0;
  };
  auto fixed = [](double p) { return (uint64_t)__builtin_rint(p * 0x1p60); };
  uint64_t r_sum = 0, p_sum = 0;
  if (o.sum && tid < a.granules) {
    const int g = chunk * a.granules + tid;
    float x[n];
    row.read(g, x);
#pragma unroll
    for (int e = 0; e < n; ++e) {
      const int i = row.first(g) + e;
      if (x[e] == -INFINITY) continue;
      const double p = whole(x[e], i);
      if (p > 0.0) {
        p_sum += fixed(p);
        r_sum += fixed(rest(p, i));
      }
    }
  }
  r_sum = block_sum<kRowWaves>(r_sum, sm_red);
  p_sum = block_sum<kRowWaves>(p_sum, sm_red);
  if (tid == 0) {
    uint64_t* at = a.r_sum + ((int64_t)b * a.chunks + chunk) * 2;
    __hip_atomic_store(at, r_sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __hip_atomic_store(at + 1, p_sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    const uint32_t before = __hip_atomic_fetch_add(a.arrived + b, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT);
    sm_int[1] = before == (uint32_t)a.chunks - 1;
  }
  __syncthreads();
  if (!sm_int[1]) return;
  if (tid == 0) {
    __hip_atomic_store(a.arrived + b, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    a.accepted[b] = kept + 1;
  }
  auto stored = [&](int c, int which) {
    return __hip_atomic_load(a.r_sum + ((int64_t)b * a.chunks + c) * 2 + which, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  };
  const float u = a.u[b];
  uint64_t all;
  int at = draw_chunk(a, u, [&](int c) { return stored(c, 0); }, sm_red, &sm_int[1], &sm_u64[0], all);
  const bool of_rest = all != 0;  // nothing left: the whole distribution
  __syncthreads();
  if (!of_rest) at = draw_chunk(a, u, [&](int c) { return stored(c, 1); }, sm_red, &sm_int[1], &sm_u64[0], all);
  int token = -1;
  if (at >= 0)
    token = draw_in_chunk<kBf16>(
        a, row, at, sm_u64[0],
        [&](float x, int i) {
          const double p = whole(x, i);
          return p > 0.0 ? fixed(of_rest ? rest(p, i) : p) : 0;
        },
        sm_red, &sm_int[2]);
  if (tid == 0) a.token[b] = token;
}

template <bool kBf16>
hipError_t launch_sample_of(const SampleArgs& a, hipStream_t stream) {
  hipLaunchKernelGGL((sample_chunk_kernel<kBf16>), dim3(a.chunks, a.batch), dim3(kChunkThreads), 0, stream, a);
  hipLaunchKernelGGL((sample_row_kernel<kBf16, true>), dim3(a.batch), dim3(kRowThreads), 0, stream, a);
  if (a.probs)
    hipLaunchKernelGGL((sample_probs_kernel<kBf16>), dim3((a.vocab + kChunkThreads - 1) / kChunkThreads, a.batch),
                       dim3(kChunkThreads), 0, stream, a);
  return hipGetLastError();
}

template <bool kBf16>
hipError_t launch_verify_of(const SampleArgs& a, hipStream_t stream) {
  const int rows = a.batch * a.rows_per_seq;
  hipLaunchKernelGGL((sample_chunk_kernel<kBf16>), dim3(a.chunks, rows), dim3(kChunkThreads), 0, stream, a);
  hipLaunchKernelGGL((sample_row_kernel<kBf16, false>), dim3(rows), dim3(kRowThreads), 0, stream, a);
  hipLaunchKernelGGL((verify_rest_kernel<kBf16>), dim3(a.chunks, a.batch), dim3(kRowThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_sample(const SampleArgs& a, bool bf16, hipStream_t stream) {
  return bf16 ? launch_sample_of<true>(a, stream) : launch_sample_of<false>(a, stream);
}
hipError_t launch_verify_sample(const SampleArgs& a, bool bf16, hipStream_t stream) {
  return bf16 ? launch_verify_of<true>(a, stream) : launch_verify_of<false>(a, stream);
}

}  // namespace dustin
