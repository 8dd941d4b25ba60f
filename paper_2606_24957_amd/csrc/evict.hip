// evict.hip -- the kept rows of a cache (selected by accumulated attention weight) to the front of another cache, or
// of the same one, with their weights and the new lengths.
#include "kv4.hpp"

namespace dustin {

constexpr int kEvictThreads = 256;    // out of place
constexpr int kEvictRunThreads = 1024;  // in place, and the weights
constexpr int kEvictRunPer = 8;

__device__ __forceinline__ int64_t evict_row(const EvictCache& c, int b, int pos, int64_t& scale) {
  if (c.page_table) {
    const int page = clampi(c.page_table[(int64_t)b * c.max_pages + (pos >> c.page_shift)], 0, c.num_pages - 1);
    const int slot = pos & ((1 << c.page_shift) - 1);
    scale = page * c.sstride_page + slot * c.sstride_n;
    return page * c.stride_page + slot * c.stride_n;
  }
  scale = b * c.sstride_b + pos * c.sstride_n;
  return b * c.stride_b + pos * c.stride_n;
}

// The weights' row (b, go): a block of entries at a time is read before it is written, so that w_out may be w: the
// positions ascend, idx[i] >= i, and what a block overwrites no later one reads.
__device__ __forceinline__ void evict_weights(const EvictArgs& a, int row) {
  const int b = row / a.groups, go = row - b * a.groups;
  const int n = clampi(a.count[row], 0, a.k_max);
  if (a.new_lens && go == 0 && threadIdx.x == 0) a.new_lens[b] = n;
  if (!a.w) return;
  const int32_t* idx = a.idx + b * a.idx_sb + go * a.idx_sg;
  const float* w = a.w + b * a.w_sb + go * a.w_sg;
  float* out = a.w_out + b * a.wo_sb + go * a.wo_sg;
  for (int i0 = 0; i0 < n; i0 += (int)blockDim.x * kEvictRunPer) {
    float x[kEvictRunPer];
#pragma unroll
    for (int j = 0; j < kEvictRunPer; ++j) {
      const int i = i0 + j * (int)blockDim.x + (int)threadIdx.x;
      x[j] = i < n ? w[clampi(idx[i], 0, a.w_len - 1)] : 0.f;
    }
    __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0): read before anyone writes
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kEvictRunPer; ++j) {
      const int i = i0 + j * (int)blockDim.x + (int)threadIdx.x;
      if (i < n) out[i] = x[j];
    }
  }
}

// Out of place: one thread moves a 16-byte chunk; consecutive threads take a row's chunks, its K and its V, then the
// next KV head (K and V rows that lie side by side are then read and written as one).  Bound by memory and, for one
// sequence, by the chain count, position, (page,) row: 8192 of 32768 positions, 8 KV heads, bf16, 18.9 us (3.5 TB/s).
// While each thread also carried the addresses of several chunks it took 22.8; with 2, 4 and 8 chunks to a thread, loaded
// before the first is stored, 24.8, 27.1 and 36.2: the more workgroups, the more of one's loads run beside another's
// stores.  Stores past the caches: 27.3.
template <int CPR>  // 16-byte chunks of a row
__global__ __launch_bounds__(kEvictThreads) void evict_kernel(EvictArgs a, uint32_t parts, uint32_t extra, int b0) {
  if (blockIdx.x < extra) {
    evict_weights(a, (int)blockIdx.x);
    return;
  }
  const uint32_t blk = blockIdx.x - extra, seq = blk / parts, part = blk - seq * parts;
  const int b = b0 + (int)seq;
  const uint32_t H = (uint32_t)a.num_kv_heads;
  const uint32_t e = part * kEvictThreads + threadIdx.x;
  const uint32_t chunk = e % CPR, r = a.caches == 2 ? e / (2 * CPR) : e / CPR;
  const int is_v = a.caches == 2 ? (e / CPR) & 1 : 0;
  const uint32_t i = r / H, h = r - i * H;
  const int go = a.groups == 1 ? 0 : (int)h;
  if (i >= (uint32_t)clampi(a.count[b * a.groups + go], 0, a.k_max)) return;
  const EvictCache &s = a.src[is_v], &d = a.dst[is_v];
  const int pos = clampi(a.idx[b * a.idx_sb + go * a.idx_sg + i], 0, s.cap_m1);
  int64_t soff, doff;
  const int64_t from = evict_row(s, b, pos, soff), to = evict_row(d, b, (int)i, doff);
  const u32x4 x = *reinterpret_cast<const u32x4*>(s.data + from + h * s.stride_h + 16 * chunk);
  *reinterpret_cast<u32x4*>(const_cast<uint8_t*>(d.data) + to + h * d.stride_h + 16 * chunk) = x;
  if (s.scales && chunk == 0) {
    const uint8_t* p = s.scales + soff + h * s.sstride_h;
    uint8_t* q = const_cast<uint8_t*>(d.scales) + doff + h * d.sstride_h;
    if (a.scale_bytes == 4) *reinterpret_cast<uint32_t*>(q) = *reinterpret_cast<const uint32_t*>(p);
    else *reinterpret_cast<uint16_t*>(q) = *reinterpret_cast<const uint16_t*>(p);
  }
}

// In place: a workgroup owns a 64-byte (or shorter) slice of every row of one (sequence, KV head, K or V) and walks
// the kept rows in order, a block at a time, each read whole before any of it is written.  The positions ascend, so
// idx[i] >= i: a block writes rows that only it and earlier blocks read.  Bound by the order: few workgroups, each with
// a block's reads, then its writes, one after the other.  Whole calls, 8 KV heads: 8192 of 32768 positions of one
// sequence 34.5 us in bf16 (64 workgroups, 2.0 TB/s; in pages 45) and 42 in 4 bits (16 workgroups, 0.4 TB/s; 51), 4096 of
// 32768 of sixteen 179 (3.0 TB/s; 191) and 62 (2.3; 65).
template <int SCH>  // 16-byte chunks of a slice
__global__ __launch_bounds__(kEvictRunThreads) void evict_in_place_kernel(EvictArgs a, uint32_t slices, uint32_t extra) {
  if (blockIdx.x < extra) {
    evict_weights(a, (int)blockIdx.x);
    return;
  }
  uint32_t blk = blockIdx.x - extra;
  const uint32_t slice = blk % slices;
  blk /= slices;
  const int is_v = a.caches == 2 ? (int)(blk & 1) : 0;
  blk /= (uint32_t)a.caches;
  const int b = (int)(blk / (uint32_t)a.num_kv_heads), h = (int)(blk % (uint32_t)a.num_kv_heads);
  const int go = a.groups == 1 ? 0 : h;
  const EvictCache& c = a.src[is_v];
  const int n = clampi(a.count[b * a.groups + go], 0, min(a.k_max, c.cap_m1 + 1));
  const int32_t* idx = a.idx + b * a.idx_sb + go * a.idx_sg;
  constexpr int kRows = kEvictRunThreads / SCH;
  const int r0 = (int)threadIdx.x / SCH, chunk = (int)threadIdx.x % SCH;
  const int64_t col = h * c.stride_h + (slice * SCH + chunk) * 16;
  const bool scales = c.scales && slice == 0 && chunk == 0;
  for (int i0 = 0; i0 < n; i0 += kRows * kEvictRunPer) {
    u32x4 x[kEvictRunPer];
    uint32_t sc[kEvictRunPer];
    int pos[kEvictRunPer];
#pragma unroll
    for (int j = 0; j < kEvictRunPer; ++j) {
      const int i = i0 + j * kRows + r0;
      pos[j] = i < n ? clampi(idx[i], 0, c.cap_m1) : i;
    }
#pragma unroll
    for (int j = 0; j < kEvictRunPer; ++j) {
      const int i = i0 + j * kRows + r0;
      if (i >= n || pos[j] == i) continue;
      int64_t soff;
      const int64_t from = evict_row(c, b, pos[j], soff);
      x[j] = *reinterpret_cast<const u32x4*>(c.data + from + col);
      if (scales) {
        const uint8_t* p = c.scales + soff + h * c.sstride_h;
        sc[j] = a.scale_bytes == 4 ? *reinterpret_cast<const uint32_t*>(p) : *reinterpret_cast<const uint16_t*>(p);
      }
    }
    __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0): read before anyone writes
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kEvictRunPer; ++j) {
      const int i = i0 + j * kRows + r0;
      if (i >= n || pos[j] == i) continue;
      int64_t doff;
      const int64_t to = evict_row(c, b, i, doff);
      *reinterpret_cast<u32x4*>(const_cast<uint8_t*>(c.data) + to + col) = x[j];
      if (scales) {
        uint8_t* p = const_cast<uint8_t*>(c.scales) + doff + h * c.sstride_h;
        if (a.scale_bytes == 4) *reinterpret_cast<uint32_t*>(p) = sc[j];
        else *reinterpret_cast<uint16_t*>(p) = (uint16_t)sc[j];
      }
    }
  }
}

hipError_t launch_evict(const EvictArgs& a, hipStream_t stream) {
  const int64_t extra = a.w || a.new_lens ? (int64_t)a.batch * a.groups : 0;
  const int cpr = a.row_bytes / 16;
  if (a.in_place) {
    const int sch = cpr < 4 ? cpr : 4;
    const int64_t slices = cpr / sch;
    const int64_t grid = extra + a.caches * (int64_t)a.batch * a.num_kv_heads * slices;
    if (grid > INT32_MAX / kEvictRunThreads) return hipErrorInvalidValue;
    if (grid == 0) return hipSuccess;
    hipLaunchKernelGGL(sch == 4 ? evict_in_place_kernel<4> : evict_in_place_kernel<2>, dim3((unsigned)grid),
                       dim3(kEvictRunThreads), 0, stream, a, (uint32_t)slices, (uint32_t)extra);
    return hipGetLastError();
  }
  const int64_t chunks = (int64_t)a.k_max * a.num_kv_heads * a.caches * cpr;  // of one sequence
  const int64_t parts = (chunks + kEvictThreads - 1) / kEvictThreads;
  const int64_t room = (INT64_C(1) << 32) / kEvictThreads - 1 - extra;  // a grid has less than 2^32 threads
  if (room < parts) return hipErrorInvalidValue;
  auto kernel = cpr == 2 ? evict_kernel<2> : cpr == 4 ? evict_kernel<4> : cpr == 8 ? evict_kernel<8> : evict_kernel<16>;
  const int64_t most = parts ? room / parts : a.batch;  // sequences
  for (int64_t b0 = 0; b0 < a.batch; b0 += most) {
    const int64_t n = a.batch - b0 < most ? a.batch - b0 : most, first = b0 == 0 ? extra : 0;
    if (first + n * parts == 0) continue;
    hipLaunchKernelGGL(kernel, dim3((unsigned)(first + n * parts)), dim3(kEvictThreads), 0, stream, a, (uint32_t)parts,
                       (uint32_t)first, (int)b0);
  }
  return hipGetLastError();
}

}  // namespace dustin
