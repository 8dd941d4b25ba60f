// What the 4-bit cache and eviction entry points hand to their kernels, under AddressSanitizer and
// UndefinedBehaviorSanitizer: built host-only together with csrc/api_kv4.hip, with the kernel launchers replaced by
// stubs that keep the arguments and return an error (so that no call touches a device).  The bounds by which the kernels
// clamp device values have to lie inside every cache of the call.  Prints one line per failed expectation and exits
// non-zero if any failed.
#include <stdio.h>
#include <string.h>

#include "../../paper_2606_24957_amd/csrc/kv4.hpp"

namespace dustin {
static Kv4RowsArgs rows_args;
static Attn4Args attn_args;
static EvictArgs evict_args;
hipError_t launch_kv4_append(const Kv4RowsArgs& a, hipStream_t) { return rows_args = a, hipErrorInvalidValue; }
hipError_t launch_kv4_read(const Kv4RowsArgs& a, hipStream_t) { return rows_args = a, hipErrorInvalidValue; }
hipError_t launch_evict(const EvictArgs& a, hipStream_t) { return evict_args = a, hipErrorInvalidValue; }
hipError_t launch_attn_kv4(const Attn4Args& a, int, bool, bool, hipStream_t) { return attn_args = a, hipErrorInvalidValue; }
}  // namespace dustin

static int failures = 0;
#define EXPECT(call, want)                                                                              \
  do {                                                                                                  \
    const long long got_ = (long long)(call), want_ = (long long)(want);                                \
    if (got_ != want_) {                                                                                \
      printf("FAIL line %d: %s -> %lld, expected %lld\n", __LINE__, #call, got_, want_);                \
      ++failures;                                                                                       \
    }                                                                                                   \
  } while (0)
#define BAD DUSTIN_ERR_INVALID_ARG
#define PASSED DUSTIN_ERR_LAUNCH  // validation let the call through to the (stubbed) launch

static char* fake(size_t off = 0) { return reinterpret_cast<char*>(0x10000) + off; }
template <class T>
static T* at(size_t off = 0) {
  return reinterpret_cast<T*>(fake(off));
}
static dustin_batch batch(int B, int max_len, int nq, bool own_counts, int k_max = 40) {
  dustin_batch bt;
  memset(&bt, 0, sizeof bt);
  bt.batch = B;
  bt.max_len = max_len;
  bt.nq_max = nq;
  bt.k_max = k_max;
  bt.seq_lens = at<int32_t>();
  bt.n_query = own_counts ? at<int32_t>() : nullptr;
  return bt;
}
static dustin_kv4 kv4(int64_t n, size_t off = 0, int H = 2) {
  dustin_kv4 c;
  memset(&c, 0, sizeof c);
  c.data = fake(off);
  c.scales = fake(off);
  c.num_kv_heads = H;
  c.head_dim = 128;
  c.stride_h = 64;
  c.stride_n = H * c.stride_h;
  c.stride_b = n * c.stride_n;
  c.scale_stride_h = 4;
  c.scale_stride_n = H * c.scale_stride_h;
  c.scale_stride_b = n * c.scale_stride_n;
  c.capacity = n;
  return c;
}
static dustin_kv4 paged4(int pages, size_t off = 0) {
  dustin_kv4 c = kv4(16, off);
  c.page_table = at<int32_t>();
  c.page_size = 16;
  c.max_pages = pages;
  c.num_pages = 30;
  c.stride_page = 16 * c.stride_n;
  c.scale_stride_page = 16 * c.scale_stride_n;
  return c;
}
static int rows(bool append, const dustin_kv4& k, const dustin_kv4& v, const dustin_batch& bt) {
  return append ? dustin_kv4_append(fake(), 2304, 256, 128, fake(), 2304, 256, 128, &k, &v, &bt, nullptr)
                : dustin_kv4_read(fake(), 2304, 256, 128, fake(), 2304, 256, 128, &k, &v, &bt, nullptr);
}
static int attn(bool sparse, const dustin_kv4& k, const dustin_kv4& v, const dustin_batch& bt, int Hq = 8,
                size_t bytes = (size_t)1 << 40) {
  return sparse ? dustin_sparse_verify_attn_kv4(fake(), 9216, 1024, 128, Hq, &k, &v, &bt, at<int32_t>(), 40, 40,
                                                at<int32_t>(), 1, 0.1f, fake(), 9216, 1024, 128, fake(), bytes, nullptr)
                : dustin_dense_verify_attn_kv4(fake(), 9216, 1024, 128, Hq, &k, &v, &bt, 0.1f, fake(), 9216, 1024, 128,
                                               fake(), bytes, nullptr);
}

int main() {
  // ---- sequences with window lengths of their own: the longest sequence may have the shortest window
  for (const bool four_pages : {false, true}) {
    const dustin_kv4 k = four_pages ? paged4(4) : kv4(64), v = four_pages ? paged4(4, 1 << 20) : kv4(64, 1 << 20);
    for (const bool second : {false, true}) {
      EXPECT(rows(second, k, v, batch(2, 63, 9, true)), PASSED);
      EXPECT(rows(second, k, v, batch(2, 64, 9, true)), PASSED);
      EXPECT(rows(second, k, v, batch(2, 65, 9, true)), BAD);
      EXPECT(rows(second, k, v, batch(2, 55, 9, false)), PASSED);
      EXPECT(rows(second, k, v, batch(2, 56, 9, false)), BAD);
      EXPECT(attn(second, k, v, batch(2, 63, 9, true)), PASSED);
      EXPECT(attn(second, k, v, batch(2, 64, 9, true)), PASSED);
      EXPECT(attn(second, k, v, batch(2, 65, 9, true)), BAD);
      EXPECT(attn(second, k, v, batch(2, 55, 9, false)), PASSED);
      EXPECT(attn(second, k, v, batch(2, 56, 9, false)), BAD);
    }
  }
  // ---- K and V of different capacity: a selected position is clamped into both
  for (const bool v_is_shorter : {false, true}) {
    const dustin_kv4 a = kv4(200), b = kv4(104, 1 << 20);
    EXPECT(attn(true, v_is_shorter ? a : b, v_is_shorter ? b : a, batch(2, 100, 4, false)), PASSED);
    EXPECT(dustin::attn_args.k.capacity, 104);
    EXPECT(dustin::attn_args.v.capacity, 104);
  }
  // ---- the workspace of a larger call serves a smaller one: fewer rows, sequences or tokens
  for (const int gs : {1, 4, 7, 8})
    for (const int B : {1, 9, 300})
      for (const int n : {0, 1, 500, 4000}) {
        const dustin_kv4 k = kv4(5000), v = kv4(5000, 1 << 20);
        for (int nq = 2; nq * gs <= 128; ++nq) {
          const size_t bytes = dustin_attn_kv4_workspace(B, 2 * gs, 2, nq, n);
          EXPECT(attn(false, k, v, batch(B, n, nq, false), 2 * gs, bytes), PASSED);
          EXPECT(attn(false, k, v, batch(B, n, nq - 1, false), 2 * gs, bytes), PASSED);
          EXPECT(attn(false, k, v, batch((B + 1) / 2, n / 2, (nq + 1) / 2, false), 2 * gs, bytes), PASSED);
          EXPECT(attn(false, k, v, batch(B, n, nq, false), 2 * gs, bytes - 1), DUSTIN_ERR_WORKSPACE);
        }
      }
  // ---- eviction of weights without a cache
  {
    auto alone = [&](const float* w, float* wo, int groups, int w_len, const int32_t* count) {
      return (int)dustin_kv_evict(nullptr, nullptr, nullptr, nullptr, 2, at<int32_t>(), 40, 40, count, groups, 40, w, 200,
                                  40, w_len, wo, 200, 40, nullptr, nullptr);
    };
    const dustin_kv4 k = kv4(200);
    EXPECT(alone(at<float>(), at<float>(), 1, 200, at<int32_t>()), PASSED);
    EXPECT(dustin::evict_args.caches, 0);
    EXPECT(alone(at<float>(), at<float>(), 5, 200, at<int32_t>()), PASSED);
    EXPECT(alone(at<float>(), at<float>(), 0, 200, at<int32_t>()), BAD);
    EXPECT(alone(nullptr, nullptr, 1, 200, at<int32_t>()), BAD);
    EXPECT(alone(at<float>(), nullptr, 1, 200, at<int32_t>()), BAD);
    EXPECT(alone(at<float>(), at<float>(), 1, 0, at<int32_t>()), BAD);
    EXPECT(alone(at<float>(), at<float>(), 1, 200, nullptr), BAD);
    EXPECT(dustin_kv4_evict(nullptr, nullptr, &k, nullptr, 2, at<int32_t>(), 40, 40, at<int32_t>(), 1, 40, at<float>(),
                            200, 40, 200, at<float>(), 200, 40, nullptr, nullptr),
           BAD);
  }
  // ---- rows of several sequences or heads are not written to one place
  {
    dustin_kv4 k = kv4(200), v = kv4(200, 1 << 20), ko = kv4(200, 2 << 20), vo = kv4(200, 3 << 20);
    auto evict = [&](const dustin_kv4& a, const dustin_kv4& b, const dustin_kv4& c, const dustin_kv4& d, int B = 2) {
      return (int)dustin_kv4_evict(&a, &b, &c, &d, B, at<int32_t>(), 40, 40, at<int32_t>(), 1, 40, nullptr, 0, 0, 0, nullptr,
                                   0, 0, nullptr, nullptr);
    };
    EXPECT(evict(k, v, ko, vo), PASSED);
    for (int what = 0; what < 4; ++what) {
      dustin_kv4 x = ko;
      int64_t* const stride[4] = {&x.stride_b, &x.scale_stride_b, &x.stride_h, &x.scale_stride_h};
      *stride[what] = 0;
      EXPECT(evict(k, v, x, vo), BAD);
      dustin_kv4 y = x;
      y.data = y.scales = fake(4 << 20);
      EXPECT(evict(y, v, ko, vo), PASSED);  // (read, they may be)
      EXPECT(evict(x, v, x, v), BAD);
      EXPECT(evict(k, v, x, vo, 1), what < 2 ? PASSED : BAD);
      EXPECT(rows(true, x, vo, batch(2, 100, 4, false)), BAD);
      EXPECT(rows(true, k, x, batch(2, 100, 4, false)), BAD);
      EXPECT(rows(true, x, vo, batch(1, 100, 4, false)), what < 2 ? PASSED : BAD);
      EXPECT(rows(false, x, vo, batch(2, 100, 4, false)), PASSED);
    }
    dustin_kv4 p = paged4(7, 2 << 20), q = paged4(7, 3 << 20);
    p.stride_b = p.scale_stride_b = q.stride_b = q.scale_stride_b = 0;  // (not used)
    EXPECT(evict(p, q, p, q), PASSED);
    EXPECT(rows(true, p, q, batch(2, 100, 4, false)), PASSED);
  }
  {  // ---- the most that one sequence may move to other caches
    dustin_kv4 k = paged4(1 << 24), v = paged4(1 << 24, 1 << 20), ko = paged4(1 << 24, 2 << 20), vo = paged4(1 << 24, 3 << 20);
    auto evict = [&](bool in_place, int k_max) {
      return (int)dustin_kv4_evict(&k, &v, in_place ? &k : &ko, in_place ? &v : &vo, 2, at<int32_t>(), 40, 40, at<int32_t>(), 1,
                                   k_max, nullptr, 0, 0, 0, nullptr, 0, 0, nullptr, nullptr);
    };
    EXPECT(evict(false, (1 << 27) - 1), PASSED);
    EXPECT(evict(false, 1 << 27), DUSTIN_ERR_UNSUPPORTED);
    EXPECT(evict(true, 1 << 27), PASSED);
  }
  printf("%s: %d failed expectations\n", failures ? "FAILED" : "ok", failures);
  return failures ? 1 : 0;
}
