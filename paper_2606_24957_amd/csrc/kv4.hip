// kv4.hip -- K and V rows into a 4-bit cache, and its rows read back as bf16.
#include "kv4.hpp"

namespace dustin {

constexpr int kKv4Threads = 256;

// Eight channels per thread, so that a block's largest magnitude is a maximum over four lanes; a workgroup belongs to
// one cache (K or V) and one sequence.  A block's scale is 2^(E - 2), E the exponent of its largest magnitude (the
// largest element then falls in [4, 8), of which (7, 8) is held as 6), and an element the nearest of the grid, the
// even code where two are as near.  Multiplying by the scale's inverse is exact.  Bound by memory where there is much to
// write (4 x 8192 rows of 4 KV heads: 67 MB read, 18 written in 23.4 us, 3.6 TB/s), by the launch for a window (16 x 5
// rows of 8 heads: 3.5 us).
template <int CPR>  // 16-byte chunks of a bf16 row
__global__ __launch_bounds__(kKv4Threads) void kv4_append_kernel(Kv4RowsArgs a, uint32_t parts, int b0) {
  const bool is_v = blockIdx.x & 1;
  const uint32_t seq = (blockIdx.x >> 1) / parts, part = (blockIdx.x >> 1) - seq * parts;
  const int b = b0 + (int)seq;
  const int T = a.dims.nq(b), N = a.dims.len(b);
  const uint32_t i = part * kKv4Threads + threadIdx.x;
  const uint32_t r = i / CPR, chunk = i % CPR;
  const uint32_t t = r / (uint32_t)a.num_kv_heads, h = r - t * (uint32_t)a.num_kv_heads;
  if (t >= (uint32_t)T) return;
  const int64_t pos = (int64_t)N + t;
  const Kv4View& c = is_v ? a.v : a.k;
  if (pos >= c.capacity) return;  // past the cache, or the page table: nothing is written
  const uint16_t* src = (is_v ? a.v_in : a.k_in) + b * (is_v ? a.v_sb : a.k_sb) + t * (is_v ? a.v_st : a.k_st) +
                        h * (is_v ? a.v_sh : a.k_sh);
  const u32x4 x = load16(src + 8 * chunk);
  float f[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    uint32_t u = (j & 1) ? x[j / 2] & 0xffff0000u : x[j / 2] << 16;
    const uint32_t mag = u & 0x7fffffffu;
    // an infinity counts as the largest finite number, a NaN as zero: a row in the cache is always finite
    if (mag >= 0x7f800000u) u = mag > 0x7f800000u ? 0u : (u & 0x80000000u) | 0x7f7f0000u;
    f[j] = __uint_as_float(u);
  }
  uint32_t big = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) big = max(big, __float_as_uint(f[j]) & 0x7fffffffu);
  big = max(big, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)big, 0xB1, 0xf, 0xf, false));  // quad_perm 1,0,3,2
  big = max(big, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)big, 0x4E, 0xf, 0xf, false));  // quad_perm 2,3,0,1
  const int e = max((int)(big >> 23) - 2, kKv4MinScale);
  const float inv = __uint_as_float((uint32_t)(254 - e) << 23);
#pragma unroll
  for (int j = 0; j < 8; ++j) f[j] = fminf(fmaxf(f[j] * inv, -6.f), 6.f);
  uint32_t codes = 0;
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, f[0], f[1], 1.f, 0);
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, f[2], f[3], 1.f, 1);
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, f[4], f[5], 1.f, 2);
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, f[6], f[7], 1.f, 3);
  const Kv4Row at = c.row(b, (int)pos);
  uint8_t* data = const_cast<uint8_t*>(c.data) + at.data + h * c.stride_h;
  uint8_t* scales = const_cast<uint8_t*>(c.scales) + at.scale + h * c.sstride_h;
  *reinterpret_cast<uint32_t*>(data + 4 * chunk) = codes;
  if ((chunk & 3) == 0) scales[chunk / 4] = (uint8_t)e;
}

// Sixteen bytes of bf16 to a thread, decoded by the conversion instructions; bound by its writes (the same 4 x 8192
// rows: 18 MB read, 67 written in 18.2 us, 4.7 TB/s).
template <int CPR>
__global__ __launch_bounds__(kKv4Threads) void kv4_read_kernel(Kv4RowsArgs a, uint32_t parts, int b0) {
  const bool is_v = blockIdx.x & 1;
  const uint32_t seq = (blockIdx.x >> 1) / parts, part = (blockIdx.x >> 1) - seq * parts;
  const int b = b0 + (int)seq;
  const int T = a.dims.nq(b), N = a.dims.len(b);
  const uint32_t i = part * kKv4Threads + threadIdx.x;
  const uint32_t r = i / CPR, chunk = i % CPR;
  const uint32_t t = r / (uint32_t)a.num_kv_heads, h = r - t * (uint32_t)a.num_kv_heads;
  if (t >= (uint32_t)T) return;
  const int64_t pos = (int64_t)N + t;
  const Kv4View& c = is_v ? a.v : a.k;
  if (pos >= c.capacity) return;
  const Kv4Row at = c.row(b, (int)pos);
  const uint32_t codes = *reinterpret_cast<const uint32_t*>(c.data + at.data + h * c.stride_h + 4 * chunk);
  const float scale = kv4_scale(c.scales[at.scale + h * c.sstride_h + chunk / 4]);
  uint16_t* dst = (is_v ? a.v_out : a.k_out) + b * (is_v ? a.v_sb : a.k_sb) + t * (is_v ? a.v_st : a.k_st) +
                  h * (is_v ? a.v_sh : a.k_sh);
  *reinterpret_cast<u32x4*>(dst + 8 * chunk) = kv4_decode8(codes, scale);
}

// One thread for each 16 bytes of bf16, workgroups over (sequence, part, K or V).
template <class Kernel>
static hipError_t launch_rows(const Kv4RowsArgs& a, Kernel kernel, hipStream_t stream) {
  const int64_t chunks = (int64_t)a.dims.nq_max * a.num_kv_heads * (a.head_dim / 8);  // of one sequence
  if (a.batch == 0 || chunks == 0) return hipSuccess;
  const int64_t parts = (chunks + kKv4Threads - 1) / kKv4Threads;
  const int64_t most = ((INT64_C(1) << 32) / kKv4Threads - 1) / (2 * parts);  // a grid has less than 2^32 threads
  if (most < 1) return hipErrorInvalidValue;
  for (int64_t b0 = 0; b0 < a.batch; b0 += most) {
    const int64_t n = a.batch - b0 < most ? a.batch - b0 : most;
    hipLaunchKernelGGL(kernel, dim3((unsigned)(2 * n * parts)), dim3(kKv4Threads), 0, stream, a, (uint32_t)parts,
                       (int)b0);
  }
  return hipGetLastError();
}

hipError_t launch_kv4_append(const Kv4RowsArgs& a, hipStream_t stream) {
  return a.head_dim == 64 ? launch_rows(a, kv4_append_kernel<8>, stream) : launch_rows(a, kv4_append_kernel<16>, stream);
}

hipError_t launch_kv4_read(const Kv4RowsArgs& a, hipStream_t stream) {
  return a.head_dim == 64 ? launch_rows(a, kv4_read_kernel<8>, stream) : launch_rows(a, kv4_read_kernel<16>, stream);
}

}  // namespace dustin
