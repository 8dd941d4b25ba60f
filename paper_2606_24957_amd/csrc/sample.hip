// sample.hip -- next tokens from logits with temperature, top-k, top-p and min-p, and drafted tokens accepted or
// rejected against the target's logits, from given random numbers.
//
// The kept set of a row is a prefix of its tokens in rank order (logit descending, index ascending): the k best, of
// those the fewest whose weights reach top_p of the sum, of those the ones whose weight is at least min_p of the
// largest.  It is described by the rank of its last token.  Three kernels:
//   chunks  every workgroup takes a piece of a row: its largest logit, the sum of its weights against that, and where
//           a filter needs it a histogram of counts and sums over eighths of octaves of the weight
//   rows    these joined, the eighth in which the kept set ends; the tokens that have to be ranked are listed: all that
//           may be kept where those are few (kSampleFew), otherwise those of the last eighth.  A short list (kPairs) is
//           ranked by comparing each token with each, a longer one by histograms of ever finer ranges; where the eighth
//           holds more than a list, one workgroup reads the row as often as it takes
//   rest    (verification) what is left of the target's distribution after the first rejected draft, and the draw
// Weights are computed in 64-bit floating point and summed as integers, so results do not depend on the order of
// work; see sample.hpp.
#include "sample.hpp"

namespace dustin {

namespace {

constexpr int kChunkThreads = 256;
constexpr int kRowThreads = 1024;
constexpr int kRowWaves = kRowThreads / kWave;
static_assert(kSamplePieces == kRowThreads, "a piece to a thread");
constexpr int kFew = kSampleFew, kList = kSampleList;
constexpr int kPairs = 128;  // tokens that are compared each with each
constexpr int kCutBin = 8 * (kSampleFrac + 1) - 1;  // first eighth that a weight below half a unit can fall in

// 2^(d + up) for -46 <= d <= 46, to within 2^-47: 2^d = 2^n 2^f, |f| <= 1/2, and the Taylor series of e^(f ln 2) to the
// 11th power (the next term is below 2^-47).  The coefficients are held in scalar registers (as literals, each would be
// moved to a register at every use).
struct Exp2 {
  double c[9];  // 1 / 11! ... 1 / 3!
  __device__ __forceinline__ Exp2() {
    double f = 1.0 / 39916800.0;
#pragma unroll
    for (int i = 0; i < 9; ++i) {
      c[i] = f;
      asm("" : "+s"(c[i]));
      f *= 11 - i;
    }
  }
  __device__ __forceinline__ double operator()(double d, int up = 0) const {
    const double n = __builtin_rint(d), t = (d - n) * 0.693147180559945309417;
    double s = c[0];
#pragma unroll
    for (int i = 1; i < 9; ++i) s = __builtin_fma(s, t, c[i]);
    s = __builtin_fma(s, t, 0.5);
    s = __builtin_fma(s, t, 1.0);
    s = __builtin_fma(s, t, 1.0);
    return __builtin_ldexp(s, (int)n + up);
  }
};

// The same by a table, for the kernel that computes most weights: 2^d = 2^e 2^(j / 32) 2^r, |r| <= 1/64, and the Taylor
// series of e^(r ln 2) to the 5th power (the next term is below 2^-48).  The table lies in LDS, an entry in two banks
// of its own; it holds 2^(44 + j / 32), so that the result comes as a multiple of 2^-44.
struct PowersOf2 {
  double at[32];
  constexpr PowersOf2() : at() {
    for (int j = 0; j < 32; ++j) {
      double t = 1.0, x = j * 0.693147180559945309417 / 32, sum = 0.0;
      for (int i = 1; i < 24; ++i) {
        sum += t;
        t *= x / i;
      }
      at[j] = sum * 0x1p44;
    }
  }
};
__device__ constexpr PowersOf2 kPowers;
struct TableExp2 {
  double c[5];  // ln2^5 / 5! ... ln2
  const double* table;
  __device__ __forceinline__ explicit TableExp2(const double* lds) : table(lds) {
    constexpr double l = 0.693147180559945309417;
    const double x[5] = {l * l * l * l * l / 120, l * l * l * l / 24, l * l * l / 6, l * l / 2, l};
#pragma unroll
    for (int i = 0; i < 5; ++i) {
      c[i] = x[i];
      asm("" : "+s"(c[i]));
    }
  }
  // 2^(44 + d) = u q, -46 <= d <= 0
  __device__ __forceinline__ double factors(double d, double& q) const {
    const double t = __builtin_fma(d, 32.0, 0x1.8p52);  // (its low bits: 32 d as an integer)
    const uint32_t k = (uint32_t)__double_as_longlong(t);
    const double r = __builtin_fma(t - 0x1.8p52, -1.0 / 32, d);
    q = c[0];
#pragma unroll
    for (int i = 1; i < 5; ++i) q = __builtin_fma(q, r, c[i]);
    q = __builtin_fma(q, r, 1.0);
    const uint64_t u = (uint64_t)__double_as_longlong(table[k & 31]) + ((uint64_t)((k & ~31u) << 15) << 32);
    return __longlong_as_double((long long)u);
  }
  __device__ __forceinline__ double operator()(double d) const {
    double q;
    const double u = factors(d, q);
    return u * q;
  }
  // ... rounded to an integer
  __device__ __forceinline__ uint64_t units(double d) const {
    double q;
    const double u = factors(d, q);
    return (uint64_t)__double_as_longlong(__builtin_fma(u, q, 0x1p52)) & 0xfffffffffffffull;
  }
};

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
  __device__ __forceinline__ bool filters() const { return !greedy && (k > 0 || p < 1.0 || m > 0.0); }
  // all that may be kept is few whatever the weights are: the histogram holds counts alone
  __device__ __forceinline__ bool counts_do() const { return k > 0 && k <= kFew / 2; }
};

// Weight of logit x in a row (or chunk) whose largest is top.
__device__ __forceinline__ double weight(const Exp2& exp2, float x, float top, double scale) {
  if (x == top) return top == -INFINITY ? 0.0 : 1.0;
  const double d = ((double)x - (double)top) * scale;
  if (!(d > -45.5)) return 0.0;
  const double w = exp2(d);
  return w < 0x1p-45 ? 0.0 : w;
}
// ... as a multiple of 2^-44 (the mantissa bits of it + 2^52).  What lies below 2^-45 is rounded to zero.
__device__ __forceinline__ double exponent_of(float x, float top, double scale) {
  double d = ((double)x - (double)top) * scale;
  if (top == INFINITY) d = x == INFINITY ? 0.0 : -46.0;
  return d >= -46.0 ? d : -46.0;  // (and where x is NaN)
}
__device__ __forceinline__ uint64_t units_of(const Exp2& exp2, float x, float top, double scale) {
  return (uint64_t)__double_as_longlong(exp2(exponent_of(x, top, scale), kSampleFrac) + 0x1p52) & 0xfffffffffffffull;
}

__device__ __forceinline__ uint64_t rank_of(float x, int i) {
  return ((uint64_t)~order_key(x) << kSampleIdxBits) | (uint32_t)i;
}
__device__ __forceinline__ float logit_of_key(uint32_t key) {
  return __uint_as_float((key & 0x80000000u) ? key & 0x7fffffffu : ~key);
}
__device__ __forceinline__ float logit_of_rank(uint64_t r) { return logit_of_key(~(uint32_t)(r >> kSampleIdxBits)); }

// Logits of the ranks from lo to hi lie in [bottom(hi), ceiling(lo)].
__device__ __forceinline__ float ceiling_of(uint64_t lo) {
  const uint32_t key = ~(uint32_t)(lo >> kSampleIdxBits);
  return key >= 0xff800000u ? INFINITY : logit_of_key(key);
}
__device__ __forceinline__ float bottom_of(uint64_t hi) {
  const uint32_t key = ~(uint32_t)(hi >> kSampleIdxBits);
  return key <= 0x007fffffu ? -INFINITY : logit_of_key(key);
}
__device__ __forceinline__ uint64_t whole_key(uint32_t key) {
  return ((uint64_t)~key << kSampleIdxBits) | (kSampleMaxVocab - 1);
}

// Eighth of an octave that a logit's weight falls in (an integer, ascending with it).
__device__ __forceinline__ double octave(float x, double scale) { return __builtin_floor((double)x * (scale * 8.0)); }

// The least key, of a row whose largest logit is top, whose logit satisfies a condition that holds from some logit on
// (of top it does), near a guess of it.
template <class Holds>
__device__ __forceinline__ uint32_t least_key(float top, double guess, Holds holds) {
  const uint32_t most = order_key(top);
  uint32_t key = order_key((float)guess);
  key = key > most || guess != guess ? most : key < 0x00800000u ? 0x00800000u : key;
  uint32_t lo = 0x007fffffu, hi = most;  // holds at hi; at lo not (or it is the least there is)
  // widening steps from the guess, then halving: a few of each
  for (uint32_t step = 2; lo < key && key < hi; step *= 8) {
    if (holds(logit_of_key(key))) {
      hi = key;
      key = hi - lo > step ? hi - step : lo;
    } else {
      lo = key;
      key = hi - lo > step ? lo + step : hi;
    }
    if (hi - lo <= 16) break;
  }
  while (hi - lo > 1) {
    const uint32_t mid = lo + (hi - lo) / 2;
    if (holds(logit_of_key(mid))) hi = mid;
    else lo = mid;
  }
  return hi;
}
// Least key in eighth of an octave j of the row, counted from its top's, or in a better one.
__device__ __forceinline__ uint32_t bin_key(float top, double scale, int j) {
  const double oct = octave(top, scale);
  return least_key(top, (oct - j) / (8.0 * scale), [&](float x) { return x == top || oct - octave(x, scale) <= j; });
}

// Values that workgroups of one launch hand to each other go past the caches.
template <class V>
__device__ __forceinline__ void put(V* p, V x) {
  __hip_atomic_store(p, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
template <class V>
__device__ __forceinline__ V get(const V* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
// Whether this workgroup is the last of n to come here (its writes by put() being complete), for every thread; the
// counter is back at zero then.
__device__ __forceinline__ bool arrive_last(uint32_t* counter, uint32_t n, int* sm) {
  __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0): the writes have reached memory
  __syncthreads();
  if (threadIdx.x == 0) {
    const uint32_t before = n == 1 ? 0 : __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    *sm = before == n - 1;
    if (before == n - 1 && n > 1) put(counter, 0u);
  }
  __syncthreads();
  return *sm;
}

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
  // The piece's bits, where it lies inside the row.
  __device__ __forceinline__ bool inside(int g) const { return first(g) >= 0 && first(g) + n <= vocab; }
  __device__ __forceinline__ u32x4 bits(int g) const {
    return *reinterpret_cast<const u32x4*>(row + (int64_t)first(g) * (kBf16 ? 2 : 4));
  }
  __device__ __forceinline__ static float of_bits(const u32x4& v, int e) {  // as it is (NaN stays NaN)
    if constexpr (kBf16) return __uint_as_float((e & 1) ? v[e / 2] & 0xffff0000u : v[e / 2] << 16);
    else return __uint_as_float(v[e]);
  }
};

__device__ __forceinline__ uint64_t shfl_xor_u64(uint64_t x, int d) {
  return (uint64_t)__shfl_xor((unsigned long long)x, d);
}
// One step of a scan over the wave in registers: x with the value that a DPP control moves here (`old` where none comes).
template <int ctrl, int rows, class Op>
__device__ __forceinline__ uint64_t dpp_step(uint64_t x, uint64_t old, Op op) {
  const uint32_t lo = __builtin_amdgcn_update_dpp((int)(uint32_t)old, (int)(uint32_t)x, ctrl, rows, 0xf, false);
  const uint32_t hi = __builtin_amdgcn_update_dpp((int)(old >> 32), (int)(x >> 32), ctrl, rows, 0xf, false);
  return op(x, ((uint64_t)hi << 32) | lo);
}
template <class Op>
__device__ __forceinline__ uint64_t wave_scan(uint64_t x, uint64_t old, Op op) {  // inclusive
  x = dpp_step<0x111, 0xf>(x, old, op);
  x = dpp_step<0x112, 0xf>(x, old, op);
  x = dpp_step<0x114, 0xf>(x, old, op);
  x = dpp_step<0x118, 0xf>(x, old, op);
  x = dpp_step<0x142, 0xa>(x, old, op);  // the rows' last lanes to the rows behind
  return dpp_step<0x143, 0xc>(x, old, op);
}
__device__ __forceinline__ uint64_t at_lane(uint64_t x, int lane) {  // (uniform lane)
  return ((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(x >> 32), lane) << 32) |
         (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)x, lane);
}
__device__ __forceinline__ uint64_t wave_scan(uint64_t x) {
  return wave_scan(x, 0, [](uint64_t p, uint64_t q) { return p + q; });
}
__device__ __forceinline__ uint64_t wave_sum(uint64_t x) { return at_lane(wave_scan(x), kWave - 1); }
__device__ __forceinline__ uint64_t wave_min(uint64_t x) {
  return at_lane(wave_scan(x, ~0ull, [](uint64_t p, uint64_t q) { return q < p ? q : p; }), kWave - 1);
}

// Inclusive sums over rows of 16 lanes.
__device__ __forceinline__ uint64_t row_scan(uint64_t x) {
  const auto add = [](uint64_t p, uint64_t q) { return p + q; };
  x = dpp_step<0x111, 0xf>(x, 0, add);
  x = dpp_step<0x112, 0xf>(x, 0, add);
  x = dpp_step<0x114, 0xf>(x, 0, add);
  return dpp_step<0x118, 0xf>(x, 0, add);
}

// Sum over a workgroup of `waves` waves, for every thread.  (The waves' sums are added up by a scan of 16 lanes: less
// code than a loop over them, and most of what these kernels execute is fetched for the one time.)
template <int waves>
__device__ __forceinline__ uint64_t block_sum(uint64_t x, uint64_t* sm) {
  static_assert(waves <= 16, "a row of lanes");
  const int lane = threadIdx.x & (kWave - 1);
  x = wave_scan(x);
  __syncthreads();
  if (lane == kWave - 1) sm[threadIdx.x / kWave] = x;
  __syncthreads();
  return at_lane(row_scan(lane < waves ? sm[lane] : 0), waves - 1);
}
// The sums of the threads before this one, and of all.
template <int waves>
__device__ __forceinline__ uint64_t block_before(uint64_t x, uint64_t* sm, uint64_t& all) {
  static_assert(waves <= 16, "a row of lanes");
  const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const uint64_t incl = wave_scan(x);
  __syncthreads();
  if (lane == kWave - 1) sm[wave] = incl;
  __syncthreads();
  const uint64_t own = lane < waves ? sm[lane] : 0, sums = row_scan(own);
  all = at_lane(sums, waves - 1);
  return at_lane(sums - own, wave) + incl - x;
}

// What a chunk's sums of weights are multiplied by to be against the row's largest logit: zero where not even its best
// token has a weight in the row (its others, against that one, may have), so that a chunk with a sum holds such a token.
__device__ __forceinline__ double rescaled(const Exp2& exp2, float c_top, float top, double scale) {
  if (c_top == top) return 1.0;
  return units_of(exp2, c_top, top, scale) ? exp2(exponent_of(c_top, top, scale)) : 0.0;
}
__device__ __forceinline__ uint64_t scaled(uint64_t sum, double factor) {
  return factor == 1.0 ? sum : (uint64_t)__builtin_rint((double)sum * factor);
}

// Both at once: the sums before this thread, and in all.
struct Two {
  uint64_t x, y;
};
template <int waves>
__device__ __forceinline__ Two block_before(Two v, Two* sm, Two& all) {
  static_assert(waves <= 16, "a row of lanes");
  const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const Two incl{wave_scan(v.x), wave_scan(v.y)};
  __syncthreads();
  if (lane == kWave - 1) sm[wave] = incl;
  __syncthreads();
  const Two own = lane < waves ? sm[lane] : Two{0, 0}, sums{row_scan(own.x), row_scan(own.y)};
  all = {at_lane(sums.x, waves - 1), at_lane(sums.y, waves - 1)};
  return {at_lane(sums.x - own.x, wave) + incl.x - v.x, at_lane(sums.y - own.y, wave) + incl.y - v.y};
}

// One read of the row: its tokens stay in LDS between the search for the largest and the weights against it.  Bound by
// 64-bit arithmetic (13 operations a weight, 5 to its bin) and the LDS additions of the histogram: 128 rows of 151936
// bf16 logits 31 us of mixed settings, 8 where only the largest is wanted (1.3 and 4.9 TB/s).
template <bool kBf16>
__global__ __launch_bounds__(kChunkThreads) void sample_chunk_kernel(SampleArgs a) {
  constexpr int n = RowReader<kBf16>::n, kMost = kRowThreads / kChunkThreads;  // pieces of a thread, at most
  constexpr int kWaves = kChunkThreads / kWave;
  // Histograms, one for a wave: the sum of tokens' weights as multiples of 2^-40 below bit kCountAt, their number from
  // there on.  (One for every eighth lane, where fewer lanes meet in a bin, took longer: the LDS leaves fewer workgroups
  // to a CU.)
  constexpr int kCountAt = 52;
  static_assert(kMost * n * kWave <= 2048 && kSampleFrac - 4 + 11 < kCountAt, "sums and counts side by side");
  __shared__ unsigned long long sm_hist[kWaves][kSampleBins];
  __shared__ u32x4 sm_piece[kRowThreads];
  __shared__ uint64_t sm_red[kWaves];
  __shared__ double sm_table[32];
  const int chunk = blockIdx.x, r = blockIdx.y, tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
  const int b = r / a.rows_per_seq, t = r - b * a.rows_per_seq;
  if (a.n_query && t >= a.n_query[b]) return;
  const RowReader<kBf16> row(a, b, t);
  const Settings s(a, b);
  const bool filters = s.filters(), sums = !s.greedy && !s.counts_do();
  if (tid < 32) sm_table[tid] = kPowers.at[tid];
  const TableExp2 exp2(sm_table);
  if (filters)
    for (int i = lane; i < kSampleBins; i += kWave) sm_hist[wave][i] = 0;
  // the chunk's best token: its largest logit, then the lowest index that has it; the pieces wait in LDS
  uint64_t best = ~0ull;
  {
    u32x4 v[kMost];
#pragma unroll
    for (int j = 0; j < kMost; ++j) {
      const int g = chunk * kSamplePieces + j * kChunkThreads + tid;
      if (row.inside(g)) {
        v[j] = row.bits(g);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[j][e] = kBf16 ? 0xff80ff80u : 0xff800000u;
        for (int e = 0; e < n; ++e) {  // the row's ends
          const int i = row.first(g) + e;
          if (i < 0 || i >= a.vocab) continue;
          const uint32_t y = __float_as_uint(row.at(i));
          if constexpr (kBf16) {
            const uint32_t keep = e & 1 ? 0xffffu : 0xffff0000u;
#pragma unroll
            for (int q = 0; q < 4; ++q)
              if (e / 2 == q) v[j][q] = (v[j][q] & keep) | (e & 1 ? y : y >> 16);
          } else {
#pragma unroll
            for (int q = 0; q < 4; ++q)
              if (e == q) v[j][q] = y;
          }
        }
      }
    }
    float big = -INFINITY;
#pragma unroll
    for (int j = 0; j < kMost; ++j) {
      sm_piece[j * kChunkThreads + tid] = v[j];
#pragma unroll
      for (int e = 0; e < n; ++e) big = fmaxf(big, row.of_bits(v[j], e));  // (fmaxf leaves NaN aside)
    }
    if (big != -INFINITY) {
#pragma unroll
      for (int j = kMost - 1; j >= 0; --j)
#pragma unroll
        for (int e = n - 1; e >= 0; --e)
          if (row.of_bits(v[j], e) == big)
            best = rank_of(big, row.first(chunk * kSamplePieces + j * kChunkThreads + tid) + e);
    }
  }
  best = wave_min(best);
  if (lane == 0) sm_red[wave] = best;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kWaves; ++w) best = sm_red[w] < best ? sm_red[w] : best;
  const float top = best == ~0ull ? -INFINITY : logit_of_rank(best);
  uint64_t sum = 0;
  if (!s.greedy && best != ~0ull) {
    const double oct = octave(top, s.scale);
#pragma unroll 1
    for (int j = 0; j < kMost; ++j) {
      const u32x4 v = sm_piece[j * kChunkThreads + tid];
      uint64_t w[n];
#pragma unroll
      for (int e = 0; e < n; ++e) {
        w[e] = sums ? exp2.units(exponent_of(row.of_bits(v, e), top, s.scale)) : 0;
        sum += w[e];
      }
      if (!filters) continue;
#pragma unroll
      for (int e = 0; e < n; ++e) {
        const float x = row.of_bits(v, e);
        const double d = x == top ? 0.0 : oct - octave(x, s.scale);
        if (sums ? w[e] != 0 : d < kSampleBins - 2)  // (not for NaN)
          atomicAdd(&sm_hist[wave][(int)d], ((w[e] + 8) >> 4) + (1ull << kCountAt));
      }
    }
  }
  sum = block_sum<kWaves>(sum, sm_red);
  const int64_t c0 = (int64_t)r * a.chunks, at = c0 + chunk;
  if (tid == 0) {
    a.c_top[at] = top;
    a.c_best[at] = best;
    a.c_sum[at] = sum;
  }
  if (filters)
    for (int i = tid; i < kSampleBins; i += kChunkThreads) {
      uint64_t h = 0;
      uint32_t c = 0;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        h += sm_hist[w][i] & ((1ull << kCountAt) - 1);
        c += (uint32_t)(sm_hist[w][i] >> kCountAt);
      }
      h <<= 4;
      if (sums) a.h_sum[at * kSampleBins + i] = h;
      a.h_cnt[at * kSampleBins + i] = c;
    }
}

// A piece that stays in registers; its tokens' logits one by one (-infinity outside the row).
template <bool kBf16>
struct Piece {
  const RowReader<kBf16>& row;
  int i0;
  bool inside;
  u32x4 bits;
  __device__ __forceinline__ Piece(const RowReader<kBf16>& r, int g)
      : row(r), i0(r.first(g)), inside(r.inside(g)), bits{0u, 0u, 0u, 0u} {
    if (inside) bits = row.bits(g);
  }
  __device__ __forceinline__ float logit(int e) const {
    constexpr int n = RowReader<kBf16>::n;
    if (!inside) return i0 + e >= 0 && i0 + e < row.vocab ? row.at(i0 + e) : -INFINITY;
    const int q = e * 4 / n;
    const uint32_t y = q < 2 ? (q == 0 ? bits[0] : bits[1]) : (q == 2 ? bits[2] : bits[3]);
    const float x = __uint_as_float(!kBf16 ? y : e & 1 ? y & 0xffff0000u : y << 16);
    return x != x ? -INFINITY : x;
  }
};

// Of the tokens of a chunk (one piece to a thread), the one at which the running sum of `value` passes `target` (the
// last with any, if none does); -1 where no token has any.
template <bool kBf16, class Value>
__device__ int draw_in_chunk(const SampleArgs& a, const RowReader<kBf16>& row, int chunk, uint64_t target, Value value,
                             uint64_t* sm, int* sm_token) {
  constexpr int n = RowReader<kBf16>::n;
  const Piece<kBf16> piece(row, chunk * kSamplePieces + (int)threadIdx.x);
  auto at = [&](int e) -> uint64_t {
    const float x = piece.logit(e);
    return x == -INFINITY ? 0 : value(x, piece.i0 + e);
  };
  uint64_t own = 0;
#pragma unroll 1
  for (int e = 0; e < n; ++e) own += at(e);
  if (threadIdx.x == 0) *sm_token = -1;
  uint64_t all;
  uint64_t run = block_before<kRowWaves>(own, sm, all);
  if (all && target >= all) target = all - 1;
  if (run <= target && target < run + own)  // one thread's tokens
#pragma unroll 1
    for (int e = 0; e < n; ++e) {
      const uint64_t v = at(e);
      if (run <= target && target < run + v) *sm_token = piece.i0 + e;
      run += v;
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

// The chunks joined, and what is left to do planned (each of a row's workgroups does this for itself: handing a plan
// over took longer); then up to `parts` workgroups list the tokens to be ranked, and the last of them ranks them and
// draws.  Bound by latency: some twenty steps between barriers, and code that is executed once and fetched for it.  128
// rows of 151936: 41 us, of which the second read of the rows is 7 to 10; one row of 32000: 15.
template <bool kBf16, bool kDraw>
__global__ __launch_bounds__(kRowThreads) void sample_row_kernel(SampleArgs a) {
  constexpr int n = RowReader<kBf16>::n;
  __shared__ uint64_t sm_rank[kList];
  __shared__ uint64_t sm_w[kList];
  __shared__ unsigned long long sm_sum[1024];  // a histogram of ranges of ranks
  __shared__ uint32_t sm_cnt[1024];
  __shared__ unsigned long long sm_chunk_sum[kSampleMaxChunks];
  __shared__ double sm_factor[kSampleMaxChunks];
  __shared__ int sm_off[kSampleMaxChunks];
  __shared__ unsigned long long sm_least[1024], sm_most[1024];  // ranks in them
  __shared__ uint64_t sm_red[kRowWaves], sm_u64[4];
  __shared__ Two sm_two[kRowWaves];
  __shared__ int sm_int[2];
  const int r = blockIdx.y, tid = threadIdx.x;
  const int b = r / a.rows_per_seq, t = r - b * a.rows_per_seq;
  if (a.n_query && t >= a.n_query[b]) return;
  const RowReader<kBf16> row(a, b, t);
  const Settings s(a, b);
  const Exp2 exp2;
  const int64_t c0 = (int64_t)r * a.chunks;
  const int pieces = kSamplePieces * a.chunks;
  const bool filters = s.filters(), sums = !s.greedy && !s.counts_do();

  // ---- the chunks joined: the row's best token, the sum of its weights, its histogram
  uint64_t best = tid < a.chunks ? a.c_best[c0 + tid] : ~0ull;
  const float c_top = tid < a.chunks ? a.c_top[c0 + tid] : -INFINITY;
  const uint64_t c_sum = sums && tid < a.chunks ? a.c_sum[c0 + tid] : 0;
  best = wave_min(best);
  if ((tid & (kWave - 1)) == 0) sm_red[tid / kWave] = best;
  sm_sum[tid] = 0;
  sm_cnt[tid] = 0;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kRowWaves; ++w) best = sm_red[w] < best ? sm_red[w] : best;
  const bool none = best == ~0ull;
  const float top = none ? -INFINITY : logit_of_rank(best);
  if (none || s.greedy) {  // nothing to draw from, or nothing to draw
    if (tid == 0 && blockIdx.x == 0) {
      a.row[r] = {none ? 0 : best, none ? 0 : 1ull << kSampleFrac, top};
      if constexpr (kDraw) a.token[b] = none ? -1 : (int)(best & (kSampleMaxVocab - 1));
    }
    return;
  }
  const double oct = octave(top, s.scale);
  uint64_t all_sum = 0;
  if (tid < a.chunks) {
    const double off = c_top == top ? 0.0 : oct - octave(c_top, s.scale);
    const double factor = rescaled(exp2, c_top, top, s.scale);
    sm_off[tid] = off < kSampleBins ? (int)off : kSampleBins;
    sm_factor[tid] = factor;
    all_sum = scaled(c_sum, factor);
    sm_chunk_sum[tid] = all_sum;
  }
  SamplePlan plan{};
  plan.mode = kRowWhole;
  plan.least = ~0ull;
  if (!filters) {
    if (blockIdx.x > 0) return;
    if constexpr (!kDraw) {
      all_sum = block_sum<kRowWaves>(all_sum, sm_red);
      if (tid == 0) a.row[r] = {~0ull, all_sum, top};
      return;
    }
    __syncthreads();
  } else {
    __syncthreads();
#pragma unroll 4
    for (int e = tid; e < a.chunks * kSampleBins; e += kRowThreads) {
      const int c = e / kSampleBins, to = e - c * kSampleBins + sm_off[c];
      const uint32_t y = a.h_cnt[c0 * kSampleBins + e];
      const uint64_t z = sums ? a.h_sum[c0 * kSampleBins + e] : 0;
      if (to >= kSampleBins || !y) continue;
      atomicAdd(&sm_cnt[to], y);
      if (sums) atomicAdd(&sm_sum[to], (unsigned long long)scaled(z, sm_factor[c]));
    }
    __syncthreads();
    const uint64_t my_cnt = tid < kSampleBins ? sm_cnt[tid] : 0, my_sum = tid < kSampleBins ? sm_sum[tid] : 0;
    if (tid == 0) sm_int[0] = kSampleBins - 1;
    Two all;
    const Two before = block_before<kRowWaves>(Two{my_cnt, my_sum}, sm_two, all);
    all_sum = all.y;
    // the eighth of an octave in which the kept set ends, by count or sum, and by min_p
    const bool by_count = s.k > 0 && (uint64_t)s.k < all.x;
    const bool count_scale = by_count || s.counts_do();
    // (without top_k or top_p it ends nowhere; the sums, multiples of 2^-40 here, may be reached before the last token)
    double target = by_count ? (double)s.k : s.counts_do() ? (double)all.x : s.p < 1.0 ? s.p * (double)all_sum : INFINITY;
    const double from = (double)(count_scale ? before.x : before.y);
    const double upto = (double)(count_scale ? before.x + my_cnt : before.y + my_sum);
    if (my_cnt && upto >= target && (from < target || tid == 0)) sm_int[0] = tid;  // one thread, or none
    __syncthreads();
    int bin = sm_int[0];
    if (s.m > 0.0) {
      plan.least = whole_key(least_key(top, (double)top + (double)__log2f((float)s.m) / s.scale,
                                       [&](float x) { return weight(exp2, x, top, s.scale) >= s.m; }));
      const float x = logit_of_rank(plan.least);
      const int bin_m = x == top ? 0 : (int)(oct - octave(x, s.scale));
      // (not where top_p is a part of the sum of the top_k: all of these are needed then)
      if (bin_m < bin && !(count_scale && s.p < 1.0)) {
        bin = bin_m;
        target = -1.0;
      }
    }
    if (tid == bin) {  // (one that only min_p names may hold no token)
      sm_u64[0] = before.x;
      sm_u64[1] = before.y;
      sm_u64[2] = my_cnt;
    }
    __syncthreads();
    const uint64_t in = sm_u64[2];
    const bool p_of_k = by_count && s.p < 1.0;  // top_p of a sum that the top_k leave
    plan.mode = sm_u64[0] + in <= kFew ? kRowFew : in <= kList && !p_of_k && !s.counts_do() ? kRowList : kRowRead;
    plan.bin = bin;
    plan.hi = whole_key(bin_key(top, s.scale, bin));
    // From here on an eighth can hold tokens without a weight, which the chunks count against their own largest logits
    // or not at all.  The list leaves them out, so that it never has more than what was counted.
    if (bin >= kCutBin)
      plan.hi = min(plan.hi, whole_key(least_key(top, (double)top - 45.0 / s.scale,
                                                 [&](float x) { return units_of(exp2, x, top, s.scale) != 0; })));
    plan.lo = plan.mode == kRowList && bin > 0 ? whole_key(bin_key(top, s.scale, bin - 1)) + 1 : 0;
    plan.before_cnt = plan.mode == kRowList ? sm_u64[0] : 0;
    plan.before_sum = plan.mode == kRowList ? sm_u64[1] : 0;
    plan.all_sum = all_sum;
    plan.target = target;
    plan.by_count = by_count;
    __syncthreads();
  }
  const bool lists = plan.mode == kRowFew || plan.mode == kRowList;
  if (!lists && blockIdx.x > 0) return;
  // calls f(rank) for every token of pieces [g0, g1) whose rank lies in [lo, hi]
  auto each = [&](int g0, int g1, uint64_t lo, uint64_t hi, auto f) {
    const float x_hi = ceiling_of(lo), x_lo = bottom_of(hi);
#pragma unroll 4
    for (int g = g0 + tid; g < g1; g += kRowThreads) {
      u32x4 v = {0u, 0u, 0u, 0u};
      uint32_t hits = 0;
      const bool inside = row.inside(g);
      if (inside) {
        v = row.bits(g);
#pragma unroll
        for (int e = 0; e < n; ++e) {
          const float x = row.of_bits(v, e);
          hits |= x >= x_lo && x <= x_hi ? 1u << e : 0u;
        }
      } else {
        const int i0 = row.first(g);
        for (int e = 0; e < n; ++e) hits |= i0 + e >= 0 && i0 + e < a.vocab ? 1u << e : 0u;
      }
      while (hits) {
        const int e = __builtin_ctz(hits), i = row.first(g) + e;
        hits &= hits - 1;
        float x;
        if (inside) {
          const int q = e * 4 / n;
          const uint32_t y = q < 2 ? (q == 0 ? v[0] : v[1]) : (q == 2 ? v[2] : v[3]);
          x = __uint_as_float(!kBf16 ? y : e & 1 ? y & 0xffff0000u : y << 16);
        } else {
          x = row.at(i);
        }
        const uint64_t c = rank_of(x, i);
        if (x != -INFINITY && c >= lo && c <= hi) f(c);
      }
    }
  };
  auto units_at = [&](uint64_t c) { return units_of(exp2, logit_of_rank(c), top, s.scale); };
  int m = 0;  // tokens in the list
  if (lists) {
    const int share = (pieces + a.parts - 1) / a.parts;
    uint64_t* list = a.list + (int64_t)r * kList;
    if (tid == 0) sm_cnt[0] = 0;
    __syncthreads();
    each(blockIdx.x * share, min(pieces, (int)(blockIdx.x + 1) * share), plan.lo, plan.hi, [&](uint64_t c) {
      const uint32_t at = atomicAdd(&sm_cnt[0], 1u);
      if (at < kList) sm_rank[at] = c;
    });
    __syncthreads();
    m = min((int)sm_cnt[0], kList);
    if (a.parts > 1) {
      if (tid == 0) sm_cnt[1] = m ? __hip_atomic_fetch_add(&a.listed[r], (uint32_t)m, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0;
      __syncthreads();
      const int base = (int)sm_cnt[1];
      for (int j = tid; j < m && base + j < kList; j += kRowThreads) put(list + base + j, sm_rank[j]);
      if (!arrive_last(&a.arrived[r], a.parts, &sm_int[0])) return;
      m = min((int)get(&a.listed[r]), kList);
      for (int j = tid; j < m; j += kRowThreads) sm_rank[j] = get(list + j);
      __syncthreads();
      if (tid == 0) put(&a.listed[r], 0u);
    }
    for (int j = tid; j < m; j += kRowThreads) sm_w[j] = units_at(sm_rank[j]);
    __syncthreads();
  }
  if (plan.mode == kRowFew && m <= kPairs) {
    // ---- few: each compared with each
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
    // (without a top_k the list need not hold all that the sum is over)
    const uint64_t z_k = s.counts_do() || plan.by_count ? block_sum<kRowWaves>(kept && part == 0 ? w : 0, sm_red) : plan.all_sum;
    if (s.p < 1.0) kept &= place == 0 || (double)before < s.p * (double)z_k;
    kept &= place == 0 || weight(exp2, logit_of_rank(c), top, s.scale) >= s.m;
    const uint64_t z = block_sum<kRowWaves>(kept && part == 0 ? w : 0, sm_red);
    if (tid == 0) sm_u64[3] = 0;
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
  uint64_t last = ~0ull;  // its rank
  auto each_token = [&](uint64_t lo, uint64_t hi, auto f) {
    if (lists) {
      for (int j = tid; j < m; j += kRowThreads)
        if (sm_rank[j] >= lo && sm_rank[j] <= hi) f(sm_rank[j], sm_w[j]);
    } else {
      each(0, pieces, lo, hi, [&](uint64_t c) { f(c, units_at(c)); });
    }
  };
  // the first token of ranks lo .. hi at which the running count (or sum), from what is before them, reaches the
  // target, else the last there is; the sum up to it
  constexpr int kCompare = 32;
  auto find_token = [&](uint64_t lo, uint64_t hi, uint64_t cnt_b, uint64_t sum_b, bool by_sum, double target,
                        uint64_t& sum) {
    for (;;) {
      const int bits = hi == lo ? 0 : 64 - __clzll((long long)(hi - lo));
      const int shift = bits > 10 ? bits - 10 : 0;
      __syncthreads();
      sm_sum[tid] = 0;
      sm_cnt[tid] = 0;
      sm_least[tid] = ~0ull;
      sm_most[tid] = 0;
      if (tid == 0) {
        sm_int[0] = -1;
        sm_int[1] = 0;
      }
      __syncthreads();
      each_token(lo, hi, [&](uint64_t c, uint64_t w) {
        if (!w) return;
        const int j = (int)((c - lo) >> shift);
        atomicAdd(&sm_cnt[j], 1u);
        atomicAdd(&sm_sum[j], (unsigned long long)w);
        atomicMin(&sm_least[j], (unsigned long long)c);
        atomicMax(&sm_most[j], (unsigned long long)c);
      });
      __syncthreads();
      const uint64_t oc = sm_cnt[tid], os = sm_sum[tid];
      Two all;
      const Two before = block_before<kRowWaves>(Two{oc, os}, sm_two, all);
      const uint64_t cb = cnt_b + before.x, sb = sum_b + before.y;
      const double from = (double)(by_sum ? sb : cb), upto = (double)(by_sum ? sb + os : cb + oc);
      if (oc && upto >= target && (from < target || before.x == 0)) sm_int[0] = tid;  // one thread, or none:
      if (oc && before.x + oc == all.x) sm_int[1] = tid;                              // then the last that has any
      __syncthreads();
      const int j = sm_int[0] < 0 ? sm_int[1] : sm_int[0];
      if (tid == j) {
        sm_u64[0] = cb;
        sm_u64[1] = sb;
        sm_u64[2] = sb + os;
      }
      __syncthreads();
      const uint32_t in = sm_cnt[j];
      cnt_b = sm_u64[0];
      sum_b = sm_u64[1];
      sum = sm_u64[2];
      lo = sm_least[j];
      hi = sm_most[j];
      if (lo >= hi) return lo;
      if (in > kCompare) continue;
      // few: each compared with each, in the histogram's place
      __syncthreads();
      if (tid == 0) {
        sm_int[0] = 0;
        sm_u64[0] = ~0ull;
        sm_u64[1] = sum;
      }
      __syncthreads();
      each_token(lo, hi, [&](uint64_t c, uint64_t w) {
        if (!w) return;
        const int at = atomicAdd(&sm_int[0], 1);
        sm_sum[at] = c;
        sm_sum[kCompare + at] = w;
      });
      __syncthreads();
      const int few = sm_int[0];
      if (tid < few) {
        const uint64_t c = sm_sum[tid], w = sm_sum[kCompare + tid];
        uint64_t cb2 = cnt_b + 1, sb2 = sum_b + w;
        uint64_t worse = 0;
        for (int i = 0; i < few; ++i) {
          const bool better = sm_sum[i] < c;
          cb2 += better;
          sb2 += better ? sm_sum[kCompare + i] : 0;
          worse += sm_sum[i] > c;
        }
        const bool reached = (by_sum ? (double)sb2 : (double)cb2) >= target || !worse;
        if (reached) atomicMin(reinterpret_cast<unsigned long long*>(&sm_u64[0]), (unsigned long long)c);
      }
      __syncthreads();
      const uint64_t found = sm_u64[0];
      if (tid < few && sm_sum[tid] == found) {
        uint64_t sb2 = sum_b;
        for (int i = 0; i < few; ++i) sb2 += sm_sum[i] <= found ? sm_sum[kCompare + i] : 0;
        sm_u64[1] = sb2;
      }
      __syncthreads();
      sum = sm_u64[1];
      return found;
    }
  };
  if (plan.mode != kRowWhole && !(plan.mode == kRowList && plan.target < 0.0)) {
    uint64_t z = plan.all_sum;  // the sum that top_p is a part of
    if (!plan.by_count && s.counts_do()) {  // fewer tokens than top_k: the list's
      uint64_t w = 0;
      for (int j = tid; j < m; j += kRowThreads) w += sm_w[j];
      z = block_sum<kRowWaves>(w, sm_red);
    }
    // all tokens that have a weight, and some without, which find_token leaves out
    const uint64_t end = lists ? plan.hi : whole_key(bin_key(top, s.scale, kSampleBins - 1));
#pragma unroll 1
    for (int by_sum = 0; by_sum < 2; ++by_sum) {  // the last of the top_k, then the last that top_p keeps
      if (by_sum ? !(s.p < 1.0) || plan.target < 0.0 : !plan.by_count) continue;
      uint64_t sum;
      const uint64_t at = find_token(lists ? plan.lo : 0, end, plan.before_cnt, plan.before_sum, by_sum,
                                     by_sum ? s.p * (double)z : (double)s.k, sum);
      last = at < last ? at : last;
      if (!by_sum) z = sum;
    }
  }
  if (plan.mode != kRowWhole && plan.least < last) last = plan.least;

  if (plan.mode == kRowFew) {
    // ---- the kept tokens are in the list: the draw by the upper and then the lower bits of their index
    constexpr int kLow = kSampleIdxBits - 10;
    uint64_t z = 0, run = 0, target = 0;
    int high = 0;
#pragma unroll
    for (int level = 0; level < 2; ++level) {
      __syncthreads();
      sm_sum[tid] = 0;
      __syncthreads();
      for (int j = tid; j < m; j += kRowThreads) {
        const int i = (int)sm_rank[j] & (kSampleMaxVocab - 1);
        if (sm_rank[j] <= last && (level == 0 || i >> kLow == high))
          atomicAdd(&sm_sum[level == 0 ? i >> kLow : i & ((1 << kLow) - 1)], (unsigned long long)sm_w[j]);
      }
      __syncthreads();
      const uint64_t w = sm_sum[tid];
      uint64_t all;
      const uint64_t before = run + block_before<kRowWaves>(w, sm_red, all);
      if (level == 0) {
        z = all;
        float u = kDraw ? a.u[b] : 0.f;
        u = u > 0.f ? u : 0.f;
        target = (uint64_t)((double)u * (double)z);
        if (target >= z) target = z - 1;
        if (tid == 0) a.row[r] = {last, z, top};
        if constexpr (!kDraw) return;
      }
      if (before <= target && target < before + w) {
        if (level == 0) {
          sm_int[0] = tid;
          sm_u64[0] = before;
        } else {
          a.token[b] = (high << kLow) + tid;
        }
      }
      __syncthreads();
      if (level == 0) {
        high = sm_int[0];
        run = sm_u64[0];
      }
    }
    return;
  }

  // ---- sums of the kept weights by chunks
  __syncthreads();
  if (plan.mode != kRowWhole && tid < a.chunks) sm_chunk_sum[tid] = 0;
  __syncthreads();
  constexpr int chunk_bits = 10 + (kBf16 ? 3 : 2);
  static_assert(1 << chunk_bits == kSamplePieces * n, "tokens of a chunk");
  if (plan.mode == kRowList) {  // (a list with all that may be kept returned above)
    for (int c = tid / kWave; c < a.chunks; c += kRowWaves) {
      uint64_t x = 0;
#pragma unroll
      for (int bin = tid & (kWave - 1); bin < kSampleBins; bin += kWave) {
        const uint64_t y = a.h_sum[(c0 + c) * kSampleBins + bin];
        x += sm_off[c] + bin < plan.bin ? scaled(y, sm_factor[c]) : 0;
      }
      x = wave_sum(x);
      if ((tid & (kWave - 1)) == 0) sm_chunk_sum[c] = x;
    }
    __syncthreads();
  }
  if (plan.mode != kRowWhole)
    each_token(0, last, [&](uint64_t c, uint64_t w) {
      const uint32_t i = (uint32_t)c & (kSampleMaxVocab - 1);
      atomicAdd(&sm_chunk_sum[(i + row.skew) >> chunk_bits], (unsigned long long)w);
    });
  __syncthreads();
  uint64_t z;
  const int chunk = draw_chunk(a, kDraw ? a.u[b] : 0.f, [&](int c) { return (uint64_t)sm_chunk_sum[c]; }, sm_red,
                               &sm_int[0], &sm_u64[0], z);
  if (tid == 0) a.row[r] = {last, z, top};
  if constexpr (kDraw) {
    if (chunk < 0) return;
    const int token = draw_in_chunk<kBf16>(
        a, row, chunk, sm_u64[0], [&](float x, int i) { return rank_of(x, i) <= last ? units_of(exp2, x, top, s.scale) : 0; }, sm_red,
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
  const Exp2 exp2;
  const SampleRow o = a.row[b];
  const float x = row.at(i);
  double p = 0.0;
  if (o.sum && x != -INFINITY && rank_of(x, i) <= o.last)
    p = weight(exp2, x, o.top, s.scale) / ((double)o.sum * 0x1p-44);
  a.probs[b * a.probs_sb + i] = (float)p;
}

// A window's accepted drafts, and a chunk's share of the distribution that the next token is drawn from; the last
// workgroup of a sequence draws it.  Bound by a chain of dependent reads (the rows' results, the drafts' logits, the
// chunk, the others' sums, the chunk that holds the token) and, where nothing is filtered, by 64-bit arithmetic: 16
// sequences of 151936 tokens with draft probabilities 21.4 us, one without 11.6 (weights by the 11th-power series over
// the sum, and draft probabilities read one after another: 24.4 and 11.5).
template <bool kBf16>
__global__ __launch_bounds__(kRowThreads) void verify_rest_kernel(SampleArgs a) {
  constexpr int n = RowReader<kBf16>::n;
  __shared__ uint64_t sm_red[kRowWaves], sm_u64[2];
  __shared__ Two sm_two[kRowWaves];
  __shared__ SampleRow sm_row;
  __shared__ double sm_table[32];
  __shared__ float sm_q[kRowThreads * (n + 1)];
  __shared__ int sm_int[3];
  const int chunk = blockIdx.x, b = blockIdx.y, tid = threadIdx.x;
  const int T = a.n_query ? clampi(a.n_query[b], 0, a.rows_per_seq) : a.rows_per_seq;
  const Settings s(a, b);
  const Exp2 exp2;
  if (T == 0) {
    if (chunk == 0 && tid == 0) {
      a.accepted[b] = 0;
      a.token[b] = -1;
    }
    return;
  }
  if (tid >= kWave && tid < kWave + 32) sm_table[tid - kWave] = kPowers.at[tid - kWave];
  // ---- accepted drafts: draft t where u q(x) < p(x), up to the first that is not
  if (tid < kWave) {
    bool ok = false;
    int x = -1;
    SampleRow o{0, 0, 0.f};
    if (tid < T) o = a.row[b * a.rows_per_seq + tid];
    if (tid < T - 1) {
      x = a.draft[b * a.draft_sb + tid];
      if (x >= 0 && x < a.vocab && o.sum) {
        const float l = RowReader<kBf16>(a, b, tid).at(x);
        const double p = l != -INFINITY && rank_of(l, x) <= o.last ? weight(exp2, l, o.top, s.scale) / ((double)o.sum * 0x1p-44) : 0.0;
        const double q = a.q ? (double)a.q[b * a.q_sb + tid * a.q_st + x] : 1.0;
        ok = (double)a.u_accept[b * a.ua_sb + tid] * q < p;
      }
    }
    const int first = min((int)__builtin_ctzll(~__ballot(ok)), T - 1);
    if (tid == first) {
      sm_int[0] = first;
      sm_int[1] = x;
      sm_row = o;
    }
  }
  __syncthreads();
  const int kept = sm_int[0];
  const bool rejected = kept < T - 1;
  const RowReader<kBf16> row(a, b, kept);
  const SampleRow o = sm_row;
  const int x_draft = sm_int[1];
  const float* q = rejected && a.q ? a.q + b * a.q_sb + kept * a.q_st : nullptr;
  const double z = 1.0 / (double)o.sum;
  const TableExp2 power(sm_table);
  // (a product with the sum's reciprocal: a bound of these rows is the rate of 64-bit arithmetic)
  auto whole = [&](float x, int i) -> double {
    const double w = rank_of(x, i) <= o.last ? power(exponent_of(x, o.top, s.scale)) : 0.0;
    return w < 0.5 ? 0.0 : w * z;
  };
  // a thread's draft probabilities, all under way at once
  float* const own_q = sm_q + tid * (n + 1);
  auto fetch_q = [&](int i0) {
    if (!q) return;
    float x[n];
    if (i0 >= 0 && i0 + n <= a.vocab) {
#pragma unroll
      for (int e = 0; e < n; ++e) x[e] = q[i0 + e];
    } else {
#pragma unroll
      for (int e = 0; e < n; ++e) x[e] = q[min(max(i0 + e, 0), a.vocab - 1)];
    }
#pragma unroll
    for (int e = 0; e < n; ++e) own_q[e] = x[e];
  };
  auto rest = [&](double p, int i0, int e) {
    if (rejected) p -= q ? (double)own_q[e] : i0 + e == x_draft ? 1.0 : 0.0;
    return p > 0.0 ? p : 0.0;
  };
  // probabilities are summed as multiples of 2^-60
  auto fixed = [](double p) { return (uint64_t)__builtin_rint(p * 0x1p60); };
  Two sum{0, 0};  // of what is left, and of the whole
  if (o.sum) {
    const Piece<kBf16> piece(row, chunk * kSamplePieces + tid);
    fetch_q(piece.i0);
    const float x_lo = bottom_of(o.last);
#pragma unroll 1
    for (int e = 0; e < n; ++e) {
      const float x = piece.logit(e);
      if (x < x_lo || x == -INFINITY) continue;
      const double p = whole(x, piece.i0 + e);
      if (p > 0.0) {
        sum.x += fixed(rest(p, piece.i0, e));
        sum.y += fixed(p);
      }
    }
  }
  Two sums;
  block_before<kRowWaves>(sum, sm_two, sums);
  if (tid == 0) {
    uint64_t* at = a.r_sum + ((int64_t)b * a.chunks + chunk) * 2;
    put(at, sums.x);
    put(at + 1, sums.y);
  }
  if (!arrive_last(&a.arrived[b], a.chunks, &sm_int[1])) return;
  if (tid == 0) a.accepted[b] = kept + 1;
  auto stored = [&](int c, int which) { return get(a.r_sum + ((int64_t)b * a.chunks + c) * 2 + which); };
  const float u = a.u[b];
  uint64_t all;
  int at = draw_chunk(a, u, [&](int c) { return stored(c, 0); }, sm_red, &sm_int[1], &sm_u64[0], all);
  const bool of_rest = all != 0;  // nothing left: the whole distribution
  __syncthreads();
  if (!of_rest) at = draw_chunk(a, u, [&](int c) { return stored(c, 1); }, sm_red, &sm_int[1], &sm_u64[0], all);
  int token = -1;
  if (at >= 0) {
    const int i0 = row.first(at * kSamplePieces + tid);
    if (at != chunk) fetch_q(i0);
    token = draw_in_chunk<kBf16>(
        a, row, at, sm_u64[0],
        [&](float x, int i) {
          const double p = whole(x, i);
          return p > 0.0 ? fixed(of_rest ? rest(p, i0, i - i0) : p) : 0;
        },
        sm_red, &sm_int[2]);
  }
  if (tid == 0) a.token[b] = token;
}

template <bool kBf16>
hipError_t launch_sample_of(const SampleArgs& a, hipStream_t stream) {
  hipLaunchKernelGGL((sample_chunk_kernel<kBf16>), dim3(a.chunks, a.batch), dim3(kChunkThreads), 0, stream, a);
  hipLaunchKernelGGL((sample_row_kernel<kBf16, true>), dim3(a.parts, a.batch), dim3(kRowThreads), 0, stream, a);
  if (a.probs)
    hipLaunchKernelGGL((sample_probs_kernel<kBf16>), dim3((a.vocab + kChunkThreads - 1) / kChunkThreads, a.batch),
                       dim3(kChunkThreads), 0, stream, a);
  return hipGetLastError();
}

template <bool kBf16>
hipError_t launch_verify_of(const SampleArgs& a, hipStream_t stream) {
  const int rows = a.batch * a.rows_per_seq;
  hipLaunchKernelGGL((sample_chunk_kernel<kBf16>), dim3(a.chunks, rows), dim3(kChunkThreads), 0, stream, a);
  hipLaunchKernelGGL((sample_row_kernel<kBf16, false>), dim3(a.parts, rows), dim3(kRowThreads), 0, stream, a);
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
