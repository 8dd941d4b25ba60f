// attn_kv4.hip -- verification attention over a 4-bit cache for gfx950: over the selected positions (sparse) or every
// committed one (dense), both followed by the causal verification window.
//
// A workgroup of four waves takes an equal share of the batch's tokens: the tokens of all (sequence, KV head) pairs
// lie end to end on one axis, in granules of 128, which is cut into as many equal runs as there are workgroups.  A run
// may end inside a pair, or span several; the parts of a pair that several workgroups hold are joined by a second
// kernel.  Within a part the waves take 32-token steps in turn:
//   K     lane (token, block) loads a block's 16 bytes, and turns them into four bf16 operands of the score product;
//         the channels of a 32-channel step are those of four blocks, and the queries are laid out to match
//   V     loads in the same way; its bf16 rows go to a wave's LDS tile, from where transpose loads take the value
//         product's operands
//   S^T = K Q^T, softmax with a lazy running maximum, O^T += V^T P^T, as in the attention over a bf16 cache.
// Two steps' rows are in flight in registers while a third is computed.
#include "kv4.hpp"

namespace dustin {

namespace {

constexpr int kD4 = 128;
constexpr int kW4 = 4;
constexpr int kStep4 = 32;
constexpr float kRescale4 = 8.f;  // lazy rescale threshold (log2)

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef short v4i16 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ u32x2 read_tr16(const char* p) {
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                       (__attribute__((address_space(3))) v4i16*)(const_cast<char*>(p))));
}

__device__ __forceinline__ uint32_t pk_bf16(float lo, float hi) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{lo, hi}, bf16x2));
}

// The run of granules of each workgroup: `first` granules of pair p, and the length of a run.
struct Plan4 {
  int64_t total, per;
};

__device__ __forceinline__ int granules_of(const Attn4Args& a, bool sparse, int pair) {
  const int b = pair / a.num_kv_heads, g = pair - b * a.num_kv_heads;
  const int T = a.dims.nq(b);
  if (T == 0) return 0;
  const int body = sparse ? clampi(a.count[b * a.groups + (a.groups == 1 ? 0 : g)], 0, a.dims.k_max) : a.dims.len(b);
  return (body + T + kAttn4Granule - 1) / kAttn4Granule;
}

// Every thread sums the granules of a run of pairs; the sums before it and in all.
__device__ __forceinline__ void scan_pairs(const Attn4Args& a, bool sparse, int64_t* sm, int& p0, int& p1, int64_t& before,
                                           int64_t& total) {
  const int per = (a.pairs + kW4 * kWave - 1) / (kW4 * kWave);
  p0 = min(a.pairs, (int)threadIdx.x * per);
  p1 = min(a.pairs, p0 + per);
  int64_t own = 0;
  for (int p = p0; p < p1; ++p) own += granules_of(a, sparse, p);
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
  int64_t incl = own;
#pragma unroll
  for (int d = 1; d < kWave; d *= 2) {
    const int64_t y = __shfl_up(incl, d);
    if (lane >= d) incl += y;
  }
  if (lane == kWave - 1) sm[wave] = incl;
  __syncthreads();
  int64_t base = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < kW4; ++w) {
    if (w < wave) base += sm[w];
    total += sm[w];
  }
  before = base + incl - own;
}

__device__ __forceinline__ int64_t run_length(const Attn4Args& a, int64_t total) {
  const int64_t per = (total + a.units - 1) / a.units;
  return per < a.min_granules ? a.min_granules : per;
}

template <int RT, bool kSparse, bool kPaged>
__global__ __launch_bounds__(kW4 * kWave) void attn_kv4_kernel(Attn4Args a) {
  constexpr int NDT = kD4 / 16;
  constexpr int kQPitch = kD4 + 8;
  constexpr int kPitch = kD4 + 4;
  constexpr bool kQReg = RT <= 3;
  constexpr int kVTile = kStep4 * kD4 * 2;
  constexpr int kBuf = RT * 16 * kPitch;  // one wave's accumulator, floats
  constexpr int kTiles = kW4 * kVTile;
  constexpr int kNB = RT <= 4 ? 2 : 1;    // of them in LDS
  constexpr int kFinal = kNB * kBuf * 4;
  __shared__ __attribute__((aligned(1024))) char smem[kTiles > kFinal ? kTiles : kFinal];
  __shared__ __attribute__((aligned(16))) uint16_t sm_q[RT * 16 * kQPitch];
  __shared__ float sm_m[kW4][RT * 16], sm_l[kW4][RT * 16];
  __shared__ int64_t sm_scan[kW4];
  __shared__ int64_t sm_first[2];

  const int lane = threadIdx.x & (kWave - 1);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int lr = lane & 15, lg = lane >> 4;
  char* const vtile = smem + wave * kVTile;

  int64_t total_g, before;
  int p0, p1;
  scan_pairs(a, kSparse, sm_scan, p0, p1, before, total_g);
  const int64_t per = run_length(a, total_g);
  const int64_t active = (total_g + per - 1) / per;  // runs there are
  // consecutive runs on one XCD: workgroups go to the XCDs in turn
  const int xcd = blockIdx.x & 7;
  const int64_t unit = (xcd * active + 7) / 8 + (blockIdx.x >> 3);
  if (unit >= ((xcd + 1) * active + 7) / 8) return;
  const int64_t start = unit * per, end = start + per < total_g ? start + per : total_g;
  for (int p = p0; p < p1; ++p) {
    const int n = granules_of(a, kSparse, p);
    if (before <= start && start < before + n) {
      sm_first[0] = p;
      sm_first[1] = before;
    }
    before += n;
  }
  __syncthreads();
  int pair = (int)sm_first[0];
  int64_t pair_g = sm_first[1];  // its first granule

  for (int64_t g0 = start; g0 < end; ++pair) {
    const int n_g = granules_of(a, kSparse, pair);
    if (n_g == 0) continue;
    const int64_t pair_end = pair_g + n_g;
    const int64_t g1 = pair_end < end ? pair_end : end;
    const int b = pair / a.num_kv_heads, g = pair - b * a.num_kv_heads, gi = a.groups == 1 ? 0 : g;
    const int N = a.dims.len(b), T = a.dims.nq(b);
    const int wstart = kSparse ? clampi(a.count[b * a.groups + gi], 0, a.dims.k_max) : N;
    const int total = wstart + T, rows = T * a.group_size;
    const int nsteps = (total + kStep4 - 1) / kStep4;
    const int s_begin = (int)(g0 - pair_g) * 4, s_end = min(nsteps, (int)(g1 - pair_g) * 4);
    const int32_t* idx_row = kSparse ? a.idx + b * a.idx_sb + gi * a.idx_sg : nullptr;
    const int cap_m1 = (int)(a.k.capacity - 1 < INT32_MAX ? a.k.capacity - 1 : INT32_MAX);
    const uint8_t* kdata = a.k.data + g * a.k.stride_h + 16 * lg;
    const uint8_t* vdata = a.v.data + g * a.v.stride_h + 16 * lg;
    const uint8_t* kscale = a.k.scales + g * a.k.sstride_h + lg;
    const uint8_t* vscale = a.v.scales + g * a.v.sstride_h + lg;

    // queries, absent rows as zeros
    __syncthreads();  // the LDS of the part before is free
    for (int e = threadIdx.x; e < RT * 16 * (kD4 / 8); e += kW4 * kWave) {
      const int r = e / (kD4 / 8), c0 = (e % (kD4 / 8)) * 8;
      u32x4 x = {0u, 0u, 0u, 0u};
      if (r < rows) {
        const int t = r / a.group_size, hh = r - t * a.group_size;
        x = load16(a.q + b * a.q_sb + t * a.q_st + (g * a.group_size + hh) * a.q_sh + c0);
      }
      *reinterpret_cast<u32x4*>(sm_q + r * kQPitch + c0) = x;
    }
    __syncthreads();
    // Q^T as B operands: lane (row lr, block lg), operand ks: channels 32 lg + 8 ks + e
    auto read_q = [&](int rt, int ks) {
      return as_bf16x8(*reinterpret_cast<const u32x4*>(sm_q + (rt * 16 + lr) * kQPitch + 32 * lg + 8 * ks));
    };
    bf16x8 qreg[kQReg ? RT : 1][4];
    if constexpr (kQReg)
#pragma unroll
      for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) qreg[rt][ks] = read_q(rt, ks);
    int limit[RT];  // token v is visible to this lane's row iff v <= limit
    float m_ref[RT];
    f32x4 acc[RT][NDT], accl[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const int r = rt * 16 + lr;
      limit[rt] = wstart + (r < rows ? r / a.group_size : T - 1);
      m_ref[rt] = -INFINITY;
      accl[rt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int dt = 0; dt < NDT; ++dt) acc[rt][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    // A step's rows pass three stages, each a load: its positions, their pages, the rows.
    struct Pos {
      int v[2];  // positions of tokens lr and 16 + lr
    };
    struct Page {
      int pos[2], page[2];
    };
    struct Rows {
      u32x4 k[2], v[2];
      uint32_t ks[2], vs[2];
    };
    auto load_pos = [&](int st) {
      Pos r;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int v = min(st * kStep4 + 16 * i + lr, total - 1);
        r.v[i] = v < wstart ? (kSparse ? idx_row[v] : v) : N + (v - wstart);
      }
      return r;
    };
    auto load_page = [&](const Pos& p) {
      Page r;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        r.pos[i] = clampi(p.v[i], 0, cap_m1);
        if constexpr (kPaged) r.page[i] = a.k.page_table[(int64_t)b * a.k.max_pages + (r.pos[i] >> a.k.page_shift)];
        else r.page[i] = b;
      }
      return r;
    };
    auto load_rows = [&](const Page& p) {
      Rows r;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        int64_t at = p.page[i], slot = p.pos[i];
        if constexpr (kPaged) {
          at = clampi(p.page[i], 0, a.k.num_pages - 1);
          slot = p.pos[i] & ((1 << a.k.page_shift) - 1);
        }
        const int64_t ko = at * (kPaged ? a.k.stride_page : a.k.stride_b) + slot * a.k.stride_n;
        const int64_t vo = at * (kPaged ? a.v.stride_page : a.v.stride_b) + slot * a.v.stride_n;
        const int64_t kso = at * (kPaged ? a.k.sstride_page : a.k.sstride_b) + slot * a.k.sstride_n;
        const int64_t vso = at * (kPaged ? a.v.sstride_page : a.v.sstride_b) + slot * a.v.sstride_n;
        r.k[i] = *reinterpret_cast<const u32x4*>(kdata + ko);
        r.v[i] = *reinterpret_cast<const u32x4*>(vdata + vo);
        r.ks[i] = kscale[kso];
        r.vs[i] = vscale[vso];
      }
      return r;
    };
    // LDS place of chunk c (8 channels) of token j of a V tile: the transpose loads of 16 tokens x 32 bytes, and the
    // stores of 16 tokens x 16 bytes, spread over all banks
    auto v_at = [&](int j, int c) { return vtile + j * 256 + 16 * (c ^ (((j & 7) << 1) | ((j >> 3) & 1))); };

    auto compute = [&](int st, const Rows& r) {
      bf16x8 kop[2][4];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float ks = kv4_scale(r.ks[i]), vs = kv4_scale(r.vs[i]);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          kop[i][w] = as_bf16x8(kv4_decode8(r.k[i][w], ks));
          *reinterpret_cast<u32x4*>(v_at(16 * i + lr, 4 * lg + w)) = kv4_decode8(r.v[i][w], vs);
        }
      }
      const int v0 = st * kStep4;
      const bool edge = v0 + kStep4 - 1 >= wstart;  // wave-uniform: masking only near the window
      bf16x8 p_op[RT];
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        f32x4 sc[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          f32x4 c = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int ks = 0; ks < 4; ++ks) {
            if constexpr (kQReg) c = mfma16x16x32(kop[i][ks], qreg[rt][ks], c);
            else c = mfma16x16x32(kop[i][ks], read_q(rt, ks), c);
          }
          sc[i] = c;
        }
        if (edge)
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (v0 + 16 * i + 4 * lg + e > min(limit[rt], total - 1)) sc[i][e] = -INFINITY;
        const float m = fmaxf(fmaxf(fmaxf(sc[0][0], sc[0][1]), fmaxf(sc[0][2], sc[0][3])),
                              fmaxf(fmaxf(sc[1][0], sc[1][1]), fmaxf(sc[1][2], sc[1][3])));
        const float mx = max_over_lane_groups(m) * a.scale_log2;
        if (__any(mx > m_ref[rt] + kRescale4)) {
          const float mn = fmaxf(m_ref[rt], mx);
          const float alpha = m_ref[rt] == -INFINITY ? 0.f : fast_exp2(m_ref[rt] - mn);
          m_ref[rt] = mn;
          accl[rt] *= alpha;
#pragma unroll
          for (int dt = 0; dt < NDT; ++dt) acc[rt][dt] *= alpha;
        }
        const float nmu = m_ref[rt] == -INFINITY ? 0.f : -m_ref[rt];
        float p[2][4];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) p[i][e] = fast_exp2(fmaf(sc[i][e], a.scale_log2, nmu));
        p_op[rt] = as_bf16x8(u32x4{pk_bf16(p[0][0], p[0][1]), pk_bf16(p[0][2], p[0][3]), pk_bf16(p[1][0], p[1][1]),
                                   pk_bf16(p[1][2], p[1][3])});
        const bf16x8 ones = as_bf16x8(u32x4{0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u});
        accl[rt] = mfma16x16x32(ones, p_op[rt], accl[rt]);
      }
      // V^T of 16 channels over the step's tokens: token 4 lg + e, and 16 + 4 lg + e
      const int j0 = 4 * lg + (lr >> 2);
#pragma unroll
      for (int dt = 0; dt < NDT; ++dt) {
        const int c = 2 * dt + ((lr >> 1) & 1);
        const u32x2 lo = read_tr16(v_at(j0, c) + 8 * (lr & 1)), hi = read_tr16(v_at(j0 + 16, c) + 8 * (lr & 1));
        const bf16x8 vt = as_bf16x8(u32x4{lo[0], lo[1], hi[0], hi[1]});
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) acc[rt][dt] = mfma16x16x32(vt, p_op[rt], acc[rt][dt]);
      }
    };

    const int st0 = s_begin + wave;
    Pos pos = load_pos(st0);
    Page page = load_page(pos);
    pos = load_pos(st0 + 4);
    Rows ra = load_rows(page);
    page = load_page(pos);
    pos = load_pos(st0 + 8);
    Rows rb = load_rows(page);
    page = load_page(pos);
    pos = load_pos(st0 + 12);
    for (int st = st0; st < s_end; st += 8) {
      compute(st, ra);
      {
        const Page now = page;
        page = load_page(pos);
        pos = load_pos(st + 16);
        ra = load_rows(now);
      }
      if (st + 4 >= s_end) break;
      compute(st + 4, rb);
      {
        const Page now = page;
        page = load_page(pos);
        pos = load_pos(st + 20);
        rb = load_rows(now);
      }
    }

    // the waves' parts become one: each at the rows' largest reference, summed in a fixed order
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
      if (lg == 0) {
        sm_m[wave][rt * 16 + lr] = m_ref[rt];
        sm_l[wave][rt * 16 + lr] = accl[rt][0];
      }
    __syncthreads();  // (and the V tiles are free)
    float* const buf = reinterpret_cast<float*>(smem);
    float beta[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const int r = rt * 16 + lr;
      const float M = fmaxf(fmaxf(sm_m[0][r], sm_m[1][r]), fmaxf(sm_m[2][r], sm_m[3][r]));
      beta[rt] = m_ref[rt] == -INFINITY ? 0.f : fast_exp2(m_ref[rt] - M);
    }
    for (int round = 0; round < kW4 / kNB; ++round) {
      if (wave / kNB == round)
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
          for (int dt = 0; dt < NDT; ++dt) {
            f32x4* at = reinterpret_cast<f32x4*>(buf + (wave % kNB) * kBuf + (rt * 16 + lr) * kPitch + 16 * dt + 4 * lg);
            const f32x4 x = acc[rt][dt] * beta[rt];
            *at = round ? *at + x : x;
          }
      __syncthreads();
    }
    const bool whole = g0 == pair_g && g1 == pair_end;
    const int64_t slot = (2 * unit + (g0 != start ? 1 : 0)) * a.rows_max;
    for (int e = threadIdx.x; e < rows * (kD4 / 8); e += kW4 * kWave) {
      const int r = e / (kD4 / 8), c0 = (e % (kD4 / 8)) * 8;
      float M = -INFINITY, L = 0.f;
#pragma unroll
      for (int w = 0; w < kW4; ++w) M = fmaxf(M, sm_m[w][r]);
#pragma unroll
      for (int w = 0; w < kW4; ++w) L += sm_m[w][r] == -INFINITY ? 0.f : sm_l[w][r] * fast_exp2(sm_m[w][r] - M);
      const float* x = buf + r * kPitch + c0;
      f32x4 lo = *reinterpret_cast<const f32x4*>(x), hi = *reinterpret_cast<const f32x4*>(x + 4);
      if constexpr (kNB == 2) {
        lo += *reinterpret_cast<const f32x4*>(x + kBuf);
        hi += *reinterpret_cast<const f32x4*>(x + kBuf + 4);
      }
      if (whole) {
        const float inv = 1.f / L;
        lo *= inv;
        hi *= inv;
        const int t = r / a.group_size, hh = r - t * a.group_size;
        *reinterpret_cast<u32x4*>(a.out + b * a.o_sb + t * a.o_st + (g * a.group_size + hh) * a.o_sh + c0) =
            u32x4{pk_bf16(lo[0], lo[1]), pk_bf16(lo[2], lo[3]), pk_bf16(hi[0], hi[1]), pk_bf16(hi[2], hi[3])};
      } else {
        float* p = a.part + (slot + r) * kD4 + c0;
        *reinterpret_cast<f32x4*>(p) = lo;
        *reinterpret_cast<f32x4*>(p + 4) = hi;
        if (c0 == 0) a.part_ml[slot + r] = make_float2(M, L);
      }
    }
    g0 = g1;
    pair_g = pair_end;
  }
}

// Joins the parts of pair blockIdx.x: 16 threads to a row, eight channels each, the parts in order.
template <bool kSparse>
__global__ __launch_bounds__(kW4 * kWave) void attn_kv4_merge_kernel(Attn4Args a) {
  __shared__ int64_t sm_scan[kW4];
  __shared__ int64_t sm_first;
  const int pair = blockIdx.x;
  int64_t total_g, before;
  int p0, p1;
  scan_pairs(a, kSparse, sm_scan, p0, p1, before, total_g);
  if (p0 <= pair && pair < p1) {
    for (int p = p0; p < pair; ++p) before += granules_of(a, kSparse, p);
    sm_first = before;
  }
  __syncthreads();
  const int64_t per = run_length(a, total_g), first = sm_first;
  const int n_g = granules_of(a, kSparse, pair);
  if (n_g == 0) return;
  const int64_t u0 = first / per, u1 = (first + n_g - 1) / per;
  if (u0 == u1) return;
  const int b = pair / a.num_kv_heads, g = pair - b * a.num_kv_heads;
  const int rows = a.dims.nq(b) * a.group_size;
  const int r = (blockIdx.y * kW4 * kWave + threadIdx.x) / 16, c0 = (threadIdx.x % 16) * 8;
  if (r >= rows) return;
  auto slot_of = [&](int64_t u) { return (2 * u + (u == u0 && u0 * per < first ? 1 : 0)) * a.rows_max + r; };
  float M = -INFINITY;
  for (int64_t u = u0; u <= u1; ++u) M = fmaxf(M, a.part_ml[slot_of(u)].x);
  f32x4 lo = {0.f, 0.f, 0.f, 0.f}, hi = lo;
  float L = 0.f;
  for (int64_t u = u0; u <= u1; ++u) {
    const int64_t s = slot_of(u);
    const float2 ml = a.part_ml[s];
    const float w = ml.x == -INFINITY ? 0.f : fast_exp2(ml.x - M);
    L += w * ml.y;
    lo += w * *reinterpret_cast<const f32x4*>(a.part + s * kD4 + c0);
    hi += w * *reinterpret_cast<const f32x4*>(a.part + s * kD4 + c0 + 4);
  }
  const float inv = 1.f / L;
  lo *= inv;
  hi *= inv;
  const int t = r / a.group_size, hh = r - t * a.group_size;
  *reinterpret_cast<u32x4*>(a.out + b * a.o_sb + t * a.o_st + (g * a.group_size + hh) * a.o_sh + c0) =
      u32x4{pk_bf16(lo[0], lo[1]), pk_bf16(lo[2], lo[3]), pk_bf16(hi[0], hi[1]), pk_bf16(hi[2], hi[3])};
}

template <bool kSparse, bool kPaged>
hipError_t launch_rt(const Attn4Args& a, int rt, hipStream_t stream) {
  const dim3 grid((unsigned)a.units), block(kW4 * kWave);
  switch (rt) {
#define CASE(n) \
  case n: hipLaunchKernelGGL((attn_kv4_kernel<n, kSparse, kPaged>), grid, block, 0, stream, a); break;
    CASE(1) CASE(2) CASE(3) CASE(4) CASE(5) CASE(6) CASE(8)
#undef CASE
    default: return hipErrorInvalidValue;
  }
  hipLaunchKernelGGL((attn_kv4_merge_kernel<kSparse>), dim3((unsigned)a.pairs, (unsigned)((a.rows_max + 15) / 16)),
                     block, 0, stream, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_attn_kv4(const Attn4Args& a, int rt, bool sparse, bool paged, hipStream_t stream) {
  if (sparse) return paged ? launch_rt<true, true>(a, rt, stream) : launch_rt<true, false>(a, rt, stream);
  return paged ? launch_rt<false, true>(a, rt, stream) : launch_rt<false, false>(a, rt, stream);
}

}  // namespace dustin
