// attn_kv4.hip -- verification attention over a 4-bit cache for gfx950: over the selected positions (sparse) or every
// committed one (dense), both followed by the causal verification window.
//
// A workgroup of eight waves takes an equal share of the batch's tokens: the tokens of all (sequence, KV head) pairs
// lie end to end on one axis, in granules of 128, which is cut into as many equal runs as there are workgroups.  A run
// may end inside a pair, or span several; the parts of a pair that several workgroups hold are joined by a second
// kernel.  A part is done in rounds of 16 tokens to a wave:
//   loads  a wave's rows of the rounds ahead go from memory straight into LDS as they are, 136 bytes a token
//   S      the wave decodes its tokens' K rows into MFMA operands (lane: token, block; the channels of one 32-channel
//          step are those of four blocks, and the queries are laid out to match): S^T = K Q^T for its tokens, all rows
//   P      probabilities against a running reference of each row, the same in all waves, as operands of the value
//          product into LDS; and its tokens' V rows, decoded, into a tile that all waves share
//   O      after the round's barrier each wave adds all the round's tokens to 16 of the 128 channels: O^T += V^T P^T
// so that a wave holds an eighth of the accumulator, and nothing is left to add up at the end but the row sums.
//
// What it does not reach is memory's rate: a token is 136 bytes and, for each 16 query rows, 16 K multiply-adds, so
// decoding, the value tile's way through LDS and the barriers of a round are in the way (with 40 rows: vector unit 44 %,
// matrix unit 27 %, LDS 40 % busy over a call).  Up to 48 query rows the registers and LDS are cut down so that two
// workgroups fit a CU, and where there is much to do (kAttn4Much) both are used: whole calls over 8 sequences of 32768
// tokens and 8 KV heads take 73 us (8 rows, 3.9 TB/s), 89 (32) and 102 (40); with one workgroup to a CU, that has two
// value tiles and more rounds in flight, these were 84, 107 and 119.  The same over 4096 selected ones (2112 granules)
// take 22, 25 and 29; there one workgroup to a CU was no slower (24, 27 and 31 for 24, 29 and 32 with two).  With more
// rows there is no room for a second: 72 rows 133 us, 88 150, 128 223; 16 sequences of 4000 to 65536 tokens, 72 rows,
// pages of 16: 293 (2.1 TB/s).
// Other forms: one value tile and two barriers a round with 72 rows 133, 88 161; the queries read from LDS as well
// 148 and 176; every wave with tokens and an accumulator of its own, joined at the end of a part, 46 where this form at
// its first took 36.
#include "kv4.hpp"

namespace dustin {

namespace {

constexpr int kD4 = 128;
constexpr int kW4 = 8;                   // waves of a workgroup: two to a SIMD
constexpr int kThreads4 = kW4 * kWave;
constexpr float kRescale4 = 8.f;         // the references move when a row's maximum passes its own by 2^8
constexpr float kNoRef = -3e38f;         // reference of a row that has seen no token: any score passes it

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef short v4i16 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) void lds_void4;

// Loads straight into LDS: lane l's 16 (or 4) bytes go to lds + 16 l (4 l).
__device__ __forceinline__ void dma16(const uint8_t* src, char* lds) {
  __builtin_amdgcn_global_load_lds(src, (lds_void4*)lds, 16, 0, 0);
}
__device__ __forceinline__ void dma4(const void* src, char* lds) {
  __builtin_amdgcn_global_load_lds(src, (lds_void4*)lds, 4, 0, 0);
}
__device__ __forceinline__ uint32_t lds_addr(const void* p) {
  return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char*)p;
}
// Waits until only the last n of the wave's loads may be outstanding.
template <int n>
__device__ __forceinline__ void wait_loads() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((n & 15) | ((n >> 4) << 14) | 0x0F70);
  asm volatile("" ::: "memory");
}
// A barrier that waits for the wave's LDS instructions but not for its loads.
__device__ __forceinline__ void lds_barrier4() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}
// Words of a ring.  (In assembly with its wait: a plain read would wait for every load in flight into LDS.)
__device__ __forceinline__ int read_word(uint32_t x) {
  int u;
  asm volatile("ds_read_b32 %0, %1\n\ts_waitcnt lgkmcnt(0)" : "=&v"(u) : "v"(x) : "memory");
  return u;
}
// The raw rows of a lane's token (K's and V's 16 bytes, their scale bytes), with n words of the rings.
template <int n>
__device__ __forceinline__ void read_raw(uint32_t rows, uint32_t scales, const uint32_t (&at)[3], u32x4& kd, u32x4& vd,
                                         uint32_t& kse, uint32_t& vse, int (&word)[3]) {
  if constexpr (n == 0) {
    asm volatile("ds_read_b128 %0, %4\n\tds_read_b128 %1, %4 offset:1024\n\tds_read_u8 %2, %5\n\t"
                 "ds_read_u8 %3, %5 offset:64\n\ts_waitcnt lgkmcnt(0)"
                 : "=&v"(kd), "=&v"(vd), "=&v"(kse), "=&v"(vse)
                 : "v"(rows), "v"(scales)
                 : "memory");
  } else if constexpr (n == 1) {
    asm volatile("ds_read_b128 %0, %5\n\tds_read_b128 %1, %5 offset:1024\n\tds_read_u8 %2, %6\n\t"
                 "ds_read_u8 %3, %6 offset:64\n\tds_read_b32 %4, %7\n\ts_waitcnt lgkmcnt(0)"
                 : "=&v"(kd), "=&v"(vd), "=&v"(kse), "=&v"(vse), "=&v"(word[0])
                 : "v"(rows), "v"(scales), "v"(at[0])
                 : "memory");
  } else {
    asm volatile("ds_read_b128 %0, %7\n\tds_read_b128 %1, %7 offset:1024\n\tds_read_u8 %2, %8\n\t"
                 "ds_read_u8 %3, %8 offset:64\n\tds_read_b32 %4, %9\n\tds_read_b32 %5, %10\n\t"
                 "ds_read_b32 %6, %11\n\ts_waitcnt lgkmcnt(0)"
                 : "=&v"(kd), "=&v"(vd), "=&v"(kse), "=&v"(vse), "=&v"(word[0]), "=&v"(word[1]), "=&v"(word[2])
                 : "v"(rows), "v"(scales), "v"(at[0]), "v"(at[1]), "v"(at[2])
                 : "memory");
  }
}

__device__ __forceinline__ u32x2 read_tr16(const char* p) {
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                       (__attribute__((address_space(3))) v4i16*)(const_cast<char*>(p))));
}

__device__ __forceinline__ uint32_t pk_bf16(float lo, float hi) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{lo, hi}, bf16x2));
}

// c + the sum of two packed bf16 numbers.
__device__ __forceinline__ float add_bf16(uint32_t two, float c) {
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, two), __builtin_bit_cast(bf16x2, 0x3f803f80u), c, false);
}

// floor(a / b) for 0 <= a < 2^22, 1 <= b < 2^22: the reciprocal's estimate is within one of it.
__device__ __forceinline__ int div22(int a, int b) {
  int q = (int)((float)a * __builtin_amdgcn_rcpf((float)b));
  q -= (int)__umul24((unsigned)q, (unsigned)b) > a ? 1 : 0;
  q += (int)__umul24((unsigned)(q + 1), (unsigned)b) <= a ? 1 : 0;
  return q;
}

// Inclusive sum over a wave (row shifts, then the rows' last lanes broadcast).
__device__ __forceinline__ int wave_sum_incl(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);
  return v;
}

// The sizes of a pair: window tokens, and tokens before them.
struct Pair4 {
  int T, body;
  __device__ __forceinline__ int granules() const {
    return T ? (body + T + kAttn4Granule - 1) / kAttn4Granule : 0;
  }
};

template <bool kSparse>
__device__ __forceinline__ Pair4 pair_of(const Attn4Args& a, int pair) {
  const int b = div22(pair, a.num_kv_heads);
  int body = 0;
  if constexpr (kSparse) body = a.count[a.groups == 1 ? b : pair];
  else body = a.dims.seq_lens[b];
  return {a.dims.nq(b), clampi(body, 0, kSparse ? a.dims.k_max : a.dims.max_len)};
}

__device__ __forceinline__ int run_length(const Attn4Args& a, int total) {
  const int units = total < kAttn4Much ? min(a.units, kAttn4Cus) : a.units;
  return max(1, (int)(((int64_t)total + units - 1) / units));
}

template <int RT, bool kSparse, bool kPaged>
__global__ __launch_bounds__(kThreads4, RT <= kAttn4Two ? 4 : 2) void attn_kv4_kernel(Attn4Args a) {
  constexpr bool kTwo = RT <= kAttn4Two;         // two workgroups to a CU
  constexpr int kTpw = 16;                       // tokens of a wave's round
  constexpr int kTok = kW4 * kTpw;               // of a round
  constexpr int kRaw = kTpw * 136;               // a wave's rows and scales of a round as they come from memory
  constexpr int kRawLoads = 3;
  constexpr int kSlots = kTwo ? 1 : RT <= 4 ? 3 : 2;  // rounds in flight
  constexpr int kAhead = kSlots == 1 ? 1 : 2;    // rounds from a position's load to its page's, and on to the rows'
  constexpr int kRing4 = kSlots == 1 ? 4 : 8;    // rounds whose positions and pages a wave holds
  // Two V tiles and two sets of probabilities, so that a round's are written while others still read those of the round
  // before: one barrier a round (where LDS holds them).  Two workgroups hide each other's second barrier.
  constexpr int kSets = !kTwo && RT <= 6 ? 2 : 1;
  constexpr int kExtra = (kSparse ? 1 : 0) + (kPaged ? 1 : 0);  // loads of positions and pages in a round
  constexpr bool kQReg = !kTwo && RT <= 6;       // the queries in registers, else read from LDS in every round
  constexpr int kQPitch = kD4 + 8;
  constexpr int kQBytes = RT * 16 * kQPitch * 2;
  constexpr int kVBytes = kTok * kD4 * 2;
  // (objects of their own: the loads in flight into one then hold back no read of another)
  static_assert(kQBytes <= kSets * kVBytes || !kQReg, "the queries pass through the V tiles");
  __shared__ __attribute__((aligned(1024))) char sm_v[kSets * kVBytes];
  __shared__ __attribute__((aligned(16))) char sm_q_own[kQReg ? 16 : kQBytes];
  __shared__ __attribute__((aligned(16))) char sm_p[kSets * RT * kTok * 32];  // [row tile][32 tokens][lane] of 16 bytes
  __shared__ __attribute__((aligned(1024))) char sm_raw[kW4 * kSlots * kRaw];
  __shared__ __attribute__((aligned(16))) char sm_pos[kSparse ? kW4 * kRing4 * kTpw * 4 : 16];
  __shared__ __attribute__((aligned(16))) char sm_page[kPaged ? kW4 * kRing4 * kTpw * 4 : 16];
  __shared__ __attribute__((aligned(16))) int sm_over[2][kW4];
  __shared__ float sm_max[kW4][RT * 16];
  __shared__ int sm_scan[kW4];
  __shared__ int sm_first[5];

  const int lane = threadIdx.x & (kWave - 1);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int lr = lane & 15, lg = lane >> 4;
  char* const raw = sm_raw + wave * kSlots * kRaw;
  char* const pos_ring = sm_pos + (kSparse ? wave * kRing4 * kTpw * 4 : 0);
  char* const page_ring = sm_page + (kPaged ? wave * kRing4 * kTpw * 4 : 0);

  // ---- the workgroup's run of granules: every thread sums those of a few pairs
  const int ppt = (a.pairs + kThreads4 - 1) / kThreads4;
  const int p0 = min(a.pairs, (int)threadIdx.x * ppt), p1 = min(a.pairs, p0 + ppt);
  int own = 0, own_T = 0, own_body = 0, own_N = 0;
  for (int p = p0; p < p1; ++p) {
    const Pair4 x = pair_of<kSparse>(a, p);
    if constexpr (kSparse) own_N = a.dims.len(div22(p, a.num_kv_heads));
    own += x.granules();
    own_T = x.T;
    own_body = x.body;
  }
  const int incl = wave_sum_incl(own);
  if (lane == kWave - 1) sm_scan[wave] = incl;
  lds_barrier4();
  int total_g = 0, before = incl - own;
#pragma unroll
  for (int w = 0; w < kW4; ++w) {
    const int x = sm_scan[w];
    before += w < wave ? x : 0;
    total_g += x;
  }
  total_g = __builtin_amdgcn_readfirstlane(total_g);
  const int per = run_length(a, total_g);
  const int active = (total_g + per - 1) / per;  // runs there are
  // consecutive runs on one XCD: workgroups go to the XCDs in turn
  const int xcd = blockIdx.x & 7;
  const int unit = (xcd * active + 7) / 8 + (blockIdx.x >> 3);
  if (unit >= ((xcd + 1) * active + 7) / 8) return;
  const int start = unit * per, end = min(total_g, start + per);
  for (int p = p0; p < p1; ++p) {
    if (ppt > 1) {
      const Pair4 x = pair_of<kSparse>(a, p);
      own = x.granules();
      own_T = x.T;
      own_body = x.body;
      own_N = a.dims.len(div22(p, a.num_kv_heads));
    }
    if (before <= start && start < before + own) {
      sm_first[0] = p;
      sm_first[1] = before;
      sm_first[2] = own_T;
      sm_first[3] = own_body;
      sm_first[4] = kSparse ? own_N : own_body;
    }
    before += own;
  }
  lds_barrier4();
  int pair = __builtin_amdgcn_readfirstlane(sm_first[0]);
  int pair_g = __builtin_amdgcn_readfirstlane(sm_first[1]);  // its first granule
  if (unit == 0 && threadIdx.x == 0) a.plan[0] = per;

  for (int g0 = start; g0 < end; ++pair) {
    const int b = div22(pair, a.num_kv_heads), g = pair - b * a.num_kv_heads;
    Pair4 pr;
    int N;
    if (g0 == start) {  // the first pair's sizes have been found
      pr.T = __builtin_amdgcn_readfirstlane(sm_first[2]);
      pr.body = __builtin_amdgcn_readfirstlane(sm_first[3]);
      N = __builtin_amdgcn_readfirstlane(sm_first[4]);
    } else {
      pr = pair_of<kSparse>(a, pair);
      N = a.dims.len(b);
    }
    const int n_g = pr.granules();
    if (n_g == 0) continue;
    const int pair_end = pair_g + n_g;
    const int g1 = min(pair_end, end);
    const int T = pr.T, wstart = pr.body, total = wstart + T, rows = T * a.group_size;
    const int t_begin = (g0 - pair_g) * kAttn4Granule, t_end = min(total, (g1 - pair_g) * kAttn4Granule);
    if (g0 == pair_g && threadIdx.x == 0) a.plan[1 + pair] = pair_g;
    const int32_t* idx_row = kSparse ? a.idx + b * a.idx_sb + (a.groups == 1 ? 0 : g) * a.idx_sg : nullptr;
    const int cap_m1 = (int)(a.k.capacity - 1);
    const uint8_t* kdata = a.k.data + g * a.k.stride_h + (kPaged ? 0 : b * a.k.stride_b) + 16 * lg;
    const uint8_t* vdata = a.v.data + g * a.v.stride_h + (kPaged ? 0 : b * a.v.stride_b) + 16 * lg;
    // scales: the first kTpw lanes take K's, the next V's
    const bool v_lane = lane & kTpw;
    const uint8_t* sdata = v_lane ? a.v.scales + g * a.v.sstride_h + (kPaged ? 0 : b * a.v.sstride_b)
                                  : a.k.scales + g * a.k.sstride_h + (kPaged ? 0 : b * a.k.sstride_b);
    const uint32_t s_sp = (uint32_t)(v_lane ? a.v.sstride_page : a.k.sstride_page);
    const uint32_t s_sn = (uint32_t)(v_lane ? a.v.sstride_n : a.k.sstride_n);

    // ---- A round's rows pass three stages, each a load into LDS: the selected positions, their pages, the rows with
    // their scales.  A token past the end is the last one, so every address is a row's.
    auto ring_of = [&](int n) { return (n & (kRing4 - 1)) * kTpw * 4; };
    auto token = [&](int n, int j) { return min(t_begin + n * kTok + wave * kTpw + j, total - 1); };
    auto load_pos = [&](int n) {
      if constexpr (kSparse)
        if (lane < kTpw) dma4(idx_row + min(token(n, lane), a.idx_last), pos_ring + ring_of(n));
    };
    auto position = [&](int v, int sel) {
      return clampi(v < wstart ? (kSparse ? sel : v) : N + (v - wstart), 0, cap_m1);
    };
    auto load_page = [&](int n, int sel) {  // sel: the round's entry `lane` of the positions
      if constexpr (kPaged)
        if (lane < kTpw)
          dma4(a.k.page_table + (int64_t)b * a.k.max_pages + (position(token(n, lane), sel) >> a.k.page_shift),
               page_ring + ring_of(n));
    };
    // (strides below 2^32: the host checks)
    auto offset = [&](int page, int slot, uint32_t sp, uint32_t sn) {
      const uint64_t o = (uint64_t)(uint32_t)slot * sn;
      return kPaged ? o + (uint64_t)(uint32_t)page * sp : o;
    };
    auto load_rows = [&](int n, int slot_n, int sel, int page) {  // sel, page: the round's entries lr
      char* const to = raw + slot_n * kRaw;
      int slot = position(token(n, lr), sel);
      if constexpr (kPaged) {
        page = clampi(page, 0, a.k.num_pages - 1);
        slot &= (1 << a.k.page_shift) - 1;
      }
      dma16(kdata + offset(page, slot, (uint32_t)a.k.stride_page, (uint32_t)a.k.stride_n), to);
      dma16(vdata + offset(page, slot, (uint32_t)a.v.stride_page, (uint32_t)a.v.stride_n), to + kTpw * 64);
      if (lane < 2 * kTpw) dma4(sdata + offset(page, slot, s_sp, s_sn), to + kTpw * 128);
    };
    const uint32_t pos_lane = lds_addr(pos_ring) + 4 * lr, page_lane = lds_addr(page_ring) + 4 * lr;
    if constexpr (kSparse) {
#pragma unroll
      for (int n = 0; n < kSlots + 2 * kAhead; ++n) load_pos(n);
    }
    // ---- queries, absent rows as zeros
    char* const sm_q = kQReg ? sm_v : sm_q_own;
    lds_barrier4();  // the LDS of the part before is free
    for (int e = threadIdx.x; e < RT * 16 * (kD4 / 8); e += kThreads4) {
      const int r = e / (kD4 / 8), c0 = (e % (kD4 / 8)) * 8;
      u32x4 x = {0u, 0u, 0u, 0u};
      if (r < rows) {
        const int t = div22(r, a.group_size), hh = r - t * a.group_size;
        x = load16(a.q + b * a.q_sb + t * a.q_st + (g * a.group_size + hh) * a.q_sh + c0);
      }
      *reinterpret_cast<u32x4*>(sm_q + (r * kQPitch + c0) * 2) = x;
    }
    if constexpr (kSparse) wait_loads<0>();
    if constexpr (kPaged) {
#pragma unroll
      for (int n = 0; n < kSlots + kAhead; ++n) load_page(n, kSparse ? read_word(pos_lane + ring_of(n)) : 0);
      wait_loads<0>();
    }
#pragma unroll
    for (int n = 0; n < kSlots; ++n)
      load_rows(n, n, kSparse ? read_word(pos_lane + ring_of(n)) : 0, kPaged ? read_word(page_lane + ring_of(n)) : 0);
    lds_barrier4();
    // (the first round's rows: no loads of positions or pages lie between it and those behind, as the loop's wait
    // counts them)
    if constexpr (kExtra > 0) wait_loads<(kSlots - 1) * kRawLoads>();
    // Q^T as B operands: lane (row lr, block lg), operand ks: channels 32 lg + 8 ks + e
    auto read_q = [&](int rt, int ks) {
      return as_bf16x8(*reinterpret_cast<const u32x4*>(sm_q + ((rt * 16 + lr) * kQPitch + 32 * lg + 8 * ks) * 2));
    };
    bf16x8 qreg[kQReg ? RT : 1][4];
    if constexpr (kQReg)
#pragma unroll
      for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) qreg[rt][ks] = read_q(rt, ks);
    if constexpr (kQReg) lds_barrier4();  // (they were in the V tiles' place)
    int limit[RT];  // token v is visible to this lane's row iff v <= limit
    float m_ref[RT], l_sum[RT];  // the row's reference (the same in every wave), and the sum over this lane's tokens
    f32x4 acc[RT];  // channels 16 wave + 4 lg + e of row lr
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const int r = rt * 16 + lr;
      limit[rt] = wstart + (r < rows ? div22(r, a.group_size) : T - 1);
      m_ref[rt] = kNoRef;
      l_sum[rt] = 0.f;
      acc[rt] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    // Place of chunk c (8 channels) of token j of the V tile: the transpose loads of 16 tokens x 32 bytes, and the
    // stores of 16 tokens x 16 bytes, spread over all banks.
    auto v_at = [&](int set, int j, int c) { return sm_v + set * kVBytes + j * 256 + 16 * (c ^ (((j & 7) << 1) | ((j >> 3) & 1))); };
    const uint32_t raw_lane = lds_addr(raw) + 16 * lane, raw_scale = lds_addr(raw) + kTpw * 128 + 4 * lr + lg;
    // this wave's probabilities in sm_p: operand bytes of its 32 tokens (or half of them)
    char* const p_own = sm_p + wave / 2 * 1024 + lane * 16 + 8 * (wave & 1);
    constexpr int kPTile = kTok / 32 * 1024;  // bytes of a row tile
    constexpr int kPSet = RT * kPTile;

    const int rounds = (t_end - t_begin + kTok - 1) / kTok;
    int slot_n = 0;
    f32x4 sc[RT];    // scores of the round whose probabilities are in LDS: tokens 4 lg + e of row lr
    u32x2 p_op[RT];  // its probabilities as operands, and their sums
    float p_sum[RT];
    auto probabilities = [&](int rt) {
      float p[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) p[e] = fast_exp2(fmaf(sc[rt][e], a.scale_log2, -m_ref[rt]));
      // bf16 operands, as the bf16 caches' attention has them; the sum is of what they are rounded to, so that an output
      // is a weighted mean of values to within 32-bit arithmetic
      p_op[rt] = u32x2{pk_bf16(p[0], p[1]), pk_bf16(p[2], p[3])};
      p_sum[rt] = add_bf16(p_op[rt][0], add_bf16(p_op[rt][1], 0.f));
    };
    auto own_max = [&](int rt) {
      return fmaxf(fmaxf(sc[rt][0], sc[rt][1]), fmaxf(sc[rt][2], sc[rt][3])) * a.scale_log2;
    };
    auto write_p = [&](int set) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) *reinterpret_cast<u32x2*>(p_own + set * kPSet + rt * kPTile) = p_op[rt];
    };
    // O^T of 16 channels: token 32 k + 4 lg + e, and 32 k + 16 + 4 lg + e
    const int j0 = 4 * lg + (lr >> 2), c_own = 2 * wave + ((lr >> 1) & 1);
    constexpr int kSteps = kTok / 32;
    bf16x8 vt[kSteps];
    auto read_v = [&](int set) {
#pragma unroll
      for (int k = 0; k < kSteps; ++k) {
        const u32x2 lo = read_tr16(v_at(set, 32 * k + j0, c_own) + 8 * (lr & 1));
        const u32x2 hi = read_tr16(v_at(set, 32 * k + j0 + 16, c_own) + 8 * (lr & 1));
        vt[k] = as_bf16x8(u32x4{lo[0], lo[1], hi[0], hi[1]});
      }
    };
    auto add_round = [&](int set) {
#pragma unroll
      for (int k = 0; k < kSteps; ++k)
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
          acc[rt] = mfma16x16x32(vt[k],
                                 as_bf16x8(*reinterpret_cast<const u32x4*>(sm_p + set * kPSet + rt * kPTile + k * 1024 +
                                                                           lane * 16)),
                                 acc[rt]);
    };
    // One turn: the values of round n - 1 are added up (its probabilities and V tile are complete: `add`), while round
    // n's rows are decoded, scored and written for the others (`next`).  Both are independent work between two
    // barriers, for the waves' latencies to hide behind each other.
    auto turn = [&](int n, bool add, bool next) {
      const int set = kSets == 2 ? n & 1 : 0, before = kSets == 2 ? set ^ 1 : 0;
      if constexpr (!kQReg) asm volatile("" ::: "memory");  // the queries stay in LDS
      if (add) read_v(before);
      if constexpr (kSets == 1) {  // one set: read it whole before it is written again
        if (add) add_round(before);
        lds_barrier4();
      }
      bf16x8 kop[4];
      if (next) {
        // this round's rows, and the positions and pages that the loads below read
        wait_loads<kSlots == 1 ? 0 : (kSlots - 1) * kRawLoads + kExtra>();
        u32x4 kd, vd;
        uint32_t kse, vse;
        const uint32_t at_sel = pos_lane + ring_of(n + kSlots), at_page = page_lane + ring_of(n + kSlots);
        const uint32_t at[3] = {kSparse ? at_sel : at_page, at_page, pos_lane + ring_of(n + kSlots + kAhead)};
        int word[3] = {0, 0, 0};
        read_raw<kSparse && kPaged ? 3 : kExtra>(raw_lane + slot_n * kRaw, raw_scale + slot_n * kRaw, at, kd, vd, kse, vse,
                                                 word);
#pragma unroll
        for (int w = 0; w < 4; ++w)
          *reinterpret_cast<u32x4*>(v_at(set, wave * kTpw + lr, 4 * lg + w)) = kv4_decode8(vd[w], kv4_scale(vse));
        load_pos(n + kSlots + 2 * kAhead);
        load_page(n + kSlots + kAhead, word[2]);
        load_rows(n + kSlots, slot_n, kSparse ? word[0] : 0, kSparse ? word[1] : word[0]);
        slot_n = slot_n + 1 == kSlots ? 0 : slot_n + 1;
#pragma unroll
        for (int w = 0; w < 4; ++w) kop[w] = as_bf16x8(kv4_decode8(kd[w], kv4_scale(kse)));
      }
      if constexpr (kSets == 2)
        if (add) add_round(before);
      if (!next) return;
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        f32x4 c = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
          if constexpr (kQReg) c = mfma16x16x32(kop[ks], qreg[rt][ks], c);
          else c = mfma16x16x32(kop[ks], read_q(rt, ks), c);
        }
        sc[rt] = c;
      }
      const int v0 = t_begin + n * kTok + wave * kTpw;
      if (v0 + kTpw - 1 >= min(wstart, t_end))  // wave-uniform: masking only near the window and the end
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (v0 + 4 * lg + e > min(limit[rt], t_end - 1)) sc[rt][e] = -INFINITY;
      bool over = false;
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        probabilities(rt);
        over |= own_max(rt) > m_ref[rt] + kRescale4;
      }
      write_p(set);
      const int any_over = __any(over) ? 1 : 0;
      if (lane == 0) sm_over[n & 1][wave] = any_over;
    };
    auto settle = [&](int n) {  // round n's probabilities are complete, against references that all waves agree on
      lds_barrier4();
      const u32x4 o0 = *reinterpret_cast<const u32x4*>(&sm_over[n & 1][0]);
      const u32x4 o1 = *reinterpret_cast<const u32x4*>(&sm_over[n & 1][4]);
      const uint32_t moves = (o0[0] | o0[1] | o0[2] | o0[3]) | (o1[0] | o1[1] | o1[2] | o1[3]);
      if (__builtin_amdgcn_readfirstlane(moves)) {
        // a row's maximum is far above its reference (in the first round, and seldom after): all references move
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
          const float m = max_over_lane_groups(own_max(rt));
          if (lg == 0) sm_max[wave][rt * 16 + lr] = m;
        }
        lds_barrier4();
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
          float mn = m_ref[rt];
#pragma unroll
          for (int w = 0; w < kW4; ++w) mn = fmaxf(mn, sm_max[w][rt * 16 + lr]);
          const float alpha = fast_exp2(m_ref[rt] - mn);
          m_ref[rt] = mn;
          l_sum[rt] *= alpha;
          acc[rt] *= alpha;
          probabilities(rt);
        }
        write_p(kSets == 2 ? n & 1 : 0);
        lds_barrier4();
      }
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) l_sum[rt] += p_sum[rt];
    };
    turn(0, false, true);
    settle(0);
    for (int n = 1; n < rounds; ++n) {
      turn(n, true, true);
      settle(n);
    }
    turn(rounds, true, false);
    wait_loads<0>();

    // ---- the rows' sums over all waves, and the outputs
    lds_barrier4();
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const float l = sum_over_lane_groups(l_sum[rt]);
      if (lg == 0) sm_max[wave][rt * 16 + lr] = l;
    }
    lds_barrier4();
    const bool whole = g0 == pair_g && g1 == pair_end;
    const int64_t part = ((int64_t)2 * unit + (g0 != start ? 1 : 0)) * a.rows_max;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const int r = rt * 16 + lr;
      float L = 0.f;
#pragma unroll
      for (int w = 0; w < kW4; ++w) L += sm_max[w][r];
      if (r >= rows) continue;
      if (whole) {
        const f32x4 x = acc[rt] * (1.f / L);
        const int t = div22(r, a.group_size), hh = r - t * a.group_size;
        *reinterpret_cast<u32x2*>(a.out + b * a.o_sb + t * a.o_st + (g * a.group_size + hh) * a.o_sh + 16 * wave +
                                  4 * lg) = u32x2{pk_bf16(x[0], x[1]), pk_bf16(x[2], x[3])};
      } else {
        *reinterpret_cast<f32x4*>(a.part + (part + r) * kD4 + 16 * wave + 4 * lg) = acc[rt];
        if (wave == 0 && lg == 0) a.part_ml[part + r] = make_float2(m_ref[rt], L);
      }
    }
    g0 = g1;
    pair_g = pair_end;
  }
}

// Joins the parts of a pair.  32 threads add up a query row's parts (four channels each), or every eighth of them where
// a pair has many parts, of which a second step adds the eight sums; always in order.  (A kernel of its own: a last
// workgroup of each pair that joins inside the first kernel would wait for the slowest of its parts.)
template <bool kSparse, bool kMany>
__global__ __launch_bounds__(256) void attn_kv4_merge_kernel(Attn4Args a) {
  __shared__ f32x4 sm_acc[kMany ? 8 : 1][32];
  __shared__ float sm_l[8];
  const int group = threadIdx.x / 32, c0 = (threadIdx.x % 32) * 4;
  const int pair = blockIdx.x, r = kMany ? blockIdx.y : blockIdx.y * 8 + group;
  const int b = div22(pair, a.num_kv_heads), g = pair - b * a.num_kv_heads;
  const Pair4 pr = pair_of<kSparse>(a, pair);
  const int per = a.plan[0], first = a.plan[1 + pair];
  const int n_g = pr.granules();
  if (n_g == 0 || r >= pr.T * a.group_size) return;
  const int u0 = first / per, u1 = (first + n_g - 1) / per;
  if (u0 == u1) return;
  auto slot_of = [&](int u) { return ((int64_t)2 * u + (u == u0 && u0 * per < first ? 1 : 0)) * a.rows_max + r; };
  float M = kNoRef;
  for (int u = u0 + (threadIdx.x & 31); u <= u1; u += 32) M = fmaxf(M, a.part_ml[slot_of(u)].x);
#pragma unroll
  for (int d = 1; d < 32; d *= 2) M = fmaxf(M, __shfl_xor(M, d));
  f32x4 x = {0.f, 0.f, 0.f, 0.f};
  float L = 0.f;
#pragma unroll 4
  for (int u = u0 + (kMany ? group : 0); u <= u1; u += kMany ? 8 : 1) {
    const int64_t s = slot_of(u);
    const float2 ml = a.part_ml[s];
    const float w = fast_exp2(ml.x - M);
    L += w * ml.y;
    x += w * *reinterpret_cast<const f32x4*>(a.part + s * kD4 + c0);
  }
  if constexpr (kMany) {
    sm_acc[group][threadIdx.x % 32] = x;
    if (c0 == 0) sm_l[group] = L;
    __syncthreads();
    if (threadIdx.x >= 32) return;
    L = sm_l[0];
    for (int i = 1; i < 8; ++i) {
      x += sm_acc[i][threadIdx.x];
      L += sm_l[i];
    }
  }
  x *= 1.f / L;
  const int t = div22(r, a.group_size), hh = r - t * a.group_size;
  *reinterpret_cast<u32x2*>(a.out + b * a.o_sb + t * a.o_st + (g * a.group_size + hh) * a.o_sh + c0) =
      u32x2{pk_bf16(x[0], x[1]), pk_bf16(x[2], x[3])};
}

template <bool kSparse, bool kPaged>
hipError_t launch_rt(const Attn4Args& a, int rt, hipStream_t stream) {
  switch (rt) {
#define CASE(n)                                                                                                  \
  case n:                                                                                                        \
    hipLaunchKernelGGL((attn_kv4_kernel<n, kSparse, kPaged>), dim3((unsigned)a.units), dim3(kThreads4), 0, stream, a); \
    break;
    CASE(1) CASE(2) CASE(3) CASE(4) CASE(5) CASE(6) CASE(8)
#undef CASE
    default: return hipErrorInvalidValue;
  }
  if (a.units > 8 * a.pairs)  // many parts to a pair (sixteen: 14.8 us for the call, without the second step 15.9)
    hipLaunchKernelGGL((attn_kv4_merge_kernel<kSparse, true>), dim3((unsigned)a.pairs, (unsigned)a.rows_max), dim3(256), 0,
                       stream, a);
  else
    hipLaunchKernelGGL((attn_kv4_merge_kernel<kSparse, false>), dim3((unsigned)a.pairs, (unsigned)(a.rows_max + 7) / 8),
                       dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_attn_kv4(const Attn4Args& a, int rt, bool sparse, bool paged, hipStream_t stream) {
  if (rt == 7) rt = 8;
  if (sparse) return paged ? launch_rt<true, true>(a, rt, stream) : launch_rt<true, false>(a, rt, stream);
  return paged ? launch_rt<false, true>(a, rt, stream) : launch_rt<false, false>(a, rt, stream);
}

}  // namespace dustin
