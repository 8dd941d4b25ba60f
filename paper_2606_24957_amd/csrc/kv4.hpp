// kv4.hpp -- the 4-bit cache: its address arithmetic and the conversions of its rows (gfx950 only).
//
// A row of d channels is d / 32 blocks of the OCP Microscaling format MXFP4: elements in E2M1 (0, 0.5, 1, 1.5, 2, 3,
// 4, 6 with a sign), two to a byte, the even channel in the low half, and for each block a scale byte e that stands
// for 2^(e - 127).  Every value a row can hold is a bf16 number, so the attention over it is bf16 arithmetic.
#pragma once

#include "kernels.hpp"

namespace dustin {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr int kKv4Block = 32;  // channels that share a scale
// Scale bytes that are written: from 2 up every value is a normal bf16 (0.5 * 2^-125 = 2^-126).
constexpr int kKv4MinScale = 2;

// Where position pos of sequence b lies: offsets of its data and scale rows (head 0), in bytes.
struct Kv4Row {
  int64_t data, scale;
};

struct Kv4View {
  const uint8_t* data;
  const uint8_t* scales;
  int64_t stride_b, stride_n, stride_h, stride_page;      // of data, in bytes
  int64_t sstride_b, sstride_n, sstride_h, sstride_page;  // of scales
  const int32_t* page_table;
  int32_t page_shift, max_pages, num_pages;
  int64_t capacity;

  // pos in [0, capacity); a page id outside the pool counts as its nearest end, for reads and for writes
  __device__ __forceinline__ int page_of(int b, int pos) const {
    return clampi(page_table[(int64_t)b * max_pages + (pos >> page_shift)], 0, num_pages - 1);
  }
  __device__ __forceinline__ Kv4Row row(int b, int pos) const {
    if (page_table) {
      const int page = page_of(b, pos), slot = pos & ((1 << page_shift) - 1);
      return {page * stride_page + slot * stride_n, page * sstride_page + slot * sstride_n};
    }
    return {b * stride_b + pos * stride_n, b * sstride_b + pos * sstride_n};
  }
};

// The scale that byte e stands for, as a float (e = 0 aside, which no written block has: its elements are zeros).
__device__ __forceinline__ float kv4_scale(uint32_t e) { return __uint_as_float(e << 23); }

// Eight elements (a dword, the first in the lowest bits) as bf16.
__device__ __forceinline__ u32x4 kv4_decode8(uint32_t codes, float scale) {
  u32x4 r;
  r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0));
  r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1));
  r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2));
  r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3));
  return r;
}

struct Kv4RowsArgs {  // append and read
  const uint16_t* k_in;
  const uint16_t* v_in;
  uint16_t* k_out;
  uint16_t* v_out;
  int64_t k_sb, k_st, k_sh, v_sb, v_st, v_sh;
  Kv4View k, v;
  SeqDims dims;
  int32_t batch, num_kv_heads, head_dim;
};
hipError_t launch_kv4_append(const Kv4RowsArgs& a, hipStream_t stream);
hipError_t launch_kv4_read(const Kv4RowsArgs& a, hipStream_t stream);

// Kept rows of a bf16 or a 4-bit cache to the front of another, or of itself (evict.hip).  A cache is described by
// byte strides; scales are NULL for bf16.
struct EvictCache {
  const uint8_t* data;
  const uint8_t* scales;
  int64_t stride_b, stride_n, stride_h, stride_page;
  int64_t sstride_b, sstride_n, sstride_h, sstride_page;
  const int32_t* page_table;
  int32_t page_shift, max_pages, num_pages;
  int32_t cap_m1;  // last addressable position
};
struct EvictArgs {
  EvictCache src[2], dst[2];  // K, V
  int32_t caches;             // 2, or 1: K alone, or 0: the weights alone
  const int32_t* idx;
  int64_t idx_sb, idx_sg;
  const int32_t* count;
  const float* w;
  float* w_out;
  int64_t w_sb, w_sg, wo_sb, wo_sg;
  int32_t* new_lens;
  int32_t batch, groups, num_kv_heads, k_max;
  int32_t w_len;         // positions of a row of w
  int32_t row_bytes, scale_bytes;
  int32_t in_place;
};
hipError_t launch_evict(const EvictArgs& a, hipStream_t stream);

// ---- verification attention over a 4-bit cache (attn_kv4.hip) ----
constexpr int kAttn4Granule = 128;  // tokens
constexpr int kAttn4Cus = 256;
constexpr int kAttn4Two = 3;        // tiles of 16 query rows up to which two workgroups share a CU
constexpr int kAttn4Much = 4096;    // granules from which on both are used

struct Attn4Args {
  const uint16_t* q;
  int64_t q_sb, q_st, q_sh;
  uint16_t* out;
  int64_t o_sb, o_st, o_sh;
  Kv4View k, v;
  SeqDims dims;
  const int32_t* idx;
  int64_t idx_sb, idx_sg;
  const int32_t* count;
  int32_t groups;
  int32_t num_kv_heads, group_size, pairs;
  float scale_log2;
  int32_t idx_last;      // last entry of a selection's row
  int32_t units;         // runs at most, a multiple of 8
  int32_t rows_max;      // query rows of a KV head, at most
  float* part;           // [units][2][rows_max][128]
  float2* part_ml;       // [units][2][rows_max]
  int32_t* plan;         // a run's length, then each pair's first granule
};
hipError_t launch_attn_kv4(const Attn4Args& a, int rt, bool sparse, bool paged, hipStream_t stream);

}  // namespace dustin
