// The host-side validation of the 4-bit cache, eviction and sampling entry points under AddressSanitizer and
// UndefinedBehaviorSanitizer: built host-only together with csrc/api_kv4.hip and csrc/api_sample.hip, with the kernel
// launchers replaced by stubs that return an error (a call that passes validation reports DUSTIN_ERR_LAUNCH and never
// touches a device).  Prints one line per failed expectation and exits non-zero if any failed.
#include <math.h>
#include <stdio.h>
#include <string.h>

#include "../../paper_2606_24957_amd/csrc/kv4.hpp"
#include "../../paper_2606_24957_amd/csrc/sample.hpp"

namespace dustin {
hipError_t launch_kv4_append(const Kv4RowsArgs&, hipStream_t) { return hipErrorInvalidValue; }
hipError_t launch_kv4_read(const Kv4RowsArgs&, hipStream_t) { return hipErrorInvalidValue; }
hipError_t launch_evict(const EvictArgs&, hipStream_t) { return hipErrorInvalidValue; }
static int last_units, last_rt;
hipError_t launch_attn_kv4(const Attn4Args& a, int rt, bool, bool, hipStream_t) {
  last_units = a.units;
  last_rt = rt;
  return hipErrorInvalidValue;
}
hipError_t launch_sample(const SampleArgs&, bool, hipStream_t) { return hipErrorInvalidValue; }
hipError_t launch_verify_sample(const SampleArgs&, bool, hipStream_t) { return hipErrorInvalidValue; }
}  // namespace dustin

static int failures = 0;
#define EXPECT(call, want)                                                                    \
  do {                                                                                        \
    const int got_ = (int)(call);                                                             \
    if (got_ != (int)(want)) {                                                                \
      printf("FAIL line %d: %s -> %d, expected %d\n", __LINE__, #call, got_, (int)(want));    \
      ++failures;                                                                             \
    }                                                                                         \
  } while (0)
#define BAD DUSTIN_ERR_INVALID_ARG
#define UNSUP DUSTIN_ERR_UNSUPPORTED
#define PASSED DUSTIN_ERR_LAUNCH  // validation let the call through to the (stubbed) launch

static char* fake(size_t off = 0) { return reinterpret_cast<char*>(0x10000) + off; }
template <class T>
static T* at(size_t off = 0) {
  return reinterpret_cast<T*>(fake(off));
}

static dustin_batch batch(int B = 2, int max_len = 100, int nq = 4, int k_max = 40) {
  dustin_batch bt;
  memset(&bt, 0, sizeof bt);
  bt.batch = B;
  bt.max_len = max_len;
  bt.nq_max = nq;
  bt.k_max = k_max;
  bt.seq_lens = at<int32_t>();
  return bt;
}

static dustin_kv4 kv4(int64_t n = 200, int H = 2, int d = 128, size_t off = 0) {
  dustin_kv4 c;
  memset(&c, 0, sizeof c);
  c.data = fake(off);
  c.scales = fake(off);
  c.num_kv_heads = H;
  c.head_dim = d;
  c.stride_h = d / 2;
  c.stride_n = H * c.stride_h;
  c.stride_b = n * c.stride_n;
  c.scale_stride_h = d / 32;
  c.scale_stride_n = H * c.scale_stride_h;
  c.scale_stride_b = n * c.scale_stride_n;
  c.capacity = n;
  return c;
}
static dustin_kv4 paged4(size_t off = 0) {
  dustin_kv4 c = kv4(16, 2, 128, off);
  c.page_table = at<int32_t>();
  c.page_size = 16;
  c.max_pages = 7;
  c.num_pages = 30;
  c.stride_page = 16 * c.stride_n;
  c.scale_stride_page = 16 * c.scale_stride_n;
  return c;
}
static dustin_kv kv16(size_t off = 0, int d = 128) {
  dustin_kv c;
  memset(&c, 0, sizeof c);
  c.data = fake(off);
  c.num_kv_heads = 2;
  c.head_dim = d;
  c.stride_h = d;
  c.stride_n = 2 * d;
  c.stride_b = 200 * 2 * d;
  c.capacity = 200;
  return c;
}

static int append(const dustin_kv4* k, const dustin_kv4* v, const dustin_batch* bt, const void* kn = fake(),
                  const void* vn = fake(), int64_t sb = 4 * 256, int64_t st = 256, int64_t sh = 128) {
  const int a = dustin_kv4_append(kn, sb, st, sh, vn, sb, st, sh, k, v, bt, nullptr);
  const int r = dustin_kv4_read(const_cast<void*>(kn), sb, st, sh, const_cast<void*>(vn), sb, st, sh, k, v, bt, nullptr);
  return a == r ? a : -1;
}
static int sparse(const dustin_kv4* k, const dustin_kv4* v, const dustin_batch* bt, int Hq = 8, const void* q = fake(),
                  void* out = fake(), const int32_t* idx = at<int32_t>(), const int32_t* count = at<int32_t>(),
                  int groups = 1, float scale = 0.1f, void* ws = fake(), size_t ws_bytes = (size_t)1 << 40,
                  int64_t sb = 4096, int64_t idx_sb = 40) {
  return dustin_sparse_verify_attn_kv4(q, sb, 1024, 128, Hq, k, v, bt, idx, idx_sb, 40, count, groups, scale, out, sb,
                                       1024, 128, ws, ws_bytes, nullptr);
}
static int dense(const dustin_kv4* k, const dustin_kv4* v, const dustin_batch* bt, int Hq = 8, void* ws = fake(),
                 size_t ws_bytes = (size_t)1 << 40, float scale = 0.1f) {
  return dustin_dense_verify_attn_kv4(fake(), 4096, 1024, 128, Hq, k, v, bt, scale, fake(), 4096, 1024, 128, ws,
                                      ws_bytes, nullptr);
}

static dustin_sampling settings() {
  dustin_sampling s;
  memset(&s, 0, sizeof s);
  s.temperature = s.top_p = 1.f;
  return s;
}
static int draw(const dustin_sampling* s, int dtype = DUSTIN_BF16, int batch = 2, int vocab = 1000,
                const void* logits = fake(), const float* u = at<float>(), int32_t* token = at<int32_t>(),
                float* probs = nullptr, int64_t probs_sb = 1000, void* ws = fake(), size_t bytes = (size_t)1 << 40,
                int64_t sb = 1000) {
  return dustin_sample(logits, dtype, sb, batch, vocab, s, u, token, probs, probs_sb, ws, bytes, nullptr);
}
static int verify(const dustin_sampling* s, int nq = 5, const int32_t* draft = at<int32_t>(),
                  const float* ua = at<float>(), int32_t* accepted = at<int32_t>(), int32_t* token = at<int32_t>(),
                  const float* q = nullptr, const int32_t* n_query = nullptr, int batch = 2,
                  size_t bytes = (size_t)1 << 40, int vocab = 1000, int64_t draft_sb = 4) {
  return dustin_verify_sample(fake(), DUSTIN_F32, 5000, 1000, batch, nq, n_query, vocab, s, draft, draft_sb, q, 4000,
                              1000, ua, 4, at<float>(), accepted, token, fake(), bytes, nullptr);
}

int main() {
  {  // ---- append and read
    const dustin_batch bt = batch();
    const dustin_kv4 k = kv4(), v = kv4(200, 2, 128, 1 << 20);
    EXPECT(append(&k, &v, &bt), PASSED);
    const dustin_kv4 k64 = kv4(200, 2, 64), p = paged4();
    EXPECT(append(&k64, &k64, &bt, fake(), fake(), 4 * 128, 128, 64), PASSED);
    EXPECT(append(&p, &p, &bt), PASSED);
    EXPECT(append(nullptr, &v, &bt), BAD);
    EXPECT(append(&k, nullptr, &bt), BAD);
    EXPECT(append(&k, &v, nullptr), BAD);
    EXPECT(append(&k, &v, &bt, nullptr), BAD);
    EXPECT(append(&k, &v, &bt, fake(), nullptr), BAD);
    EXPECT(append(&k, &v, &bt, fake(2)), BAD);
    EXPECT(append(&k, &v, &bt, fake(), fake(), 4 * 256, 252), BAD);
    dustin_batch b2 = batch(2, 197);
    EXPECT(append(&k, &v, &b2), BAD);  // 201 positions of 200
    b2 = batch(2, 196);
    EXPECT(append(&k, &v, &b2), PASSED);
    b2 = batch(2, 109);
    EXPECT(append(&p, &p, &b2), BAD);  // 113 of 7 pages
    b2 = batch(-1);
    EXPECT(append(&k, &v, &b2), BAD);
    b2 = batch();
    b2.seq_lens = nullptr;
    EXPECT(append(&k, &v, &b2), BAD);
    b2 = batch(2, INT32_MAX, INT32_MAX);
    dustin_kv4 big = kv4();
    big.capacity = (int64_t)1 << 40;
    EXPECT(append(&big, &big, &b2), UNSUP);
    big.capacity = INT32_MAX;
    b2 = batch(2, 0, INT32_MAX);
    EXPECT(append(&big, &big, &b2), UNSUP);
    for (int what = 0; what < 18; ++what) {
      dustin_kv4 x = what < 12 ? kv4() : paged4();
      int want = BAD;
      switch (what) {
        case 0: x.data = nullptr; break;
        case 1: x.scales = nullptr; break;
        case 2: x.data = fake(8); break;
        case 3: x.scales = fake(2); break;
        case 4: x.stride_n += 8; break;
        case 5: x.scale_stride_n += 2; break;
        case 6: x.stride_n = 0; break;
        case 7: x.scale_stride_n = 0; break;
        case 8: x.num_kv_heads = 0; break;
        case 9: x.capacity = 0; break;
        case 10: x.head_dim = 96; want = UNSUP; break;
        case 11: x.stride_b = -16; break;
        case 12: x.page_size = 12; break;
        case 13: x.max_pages = 0; break;
        case 14: x.num_pages = 0; break;
        case 15: x.stride_page = 0; break;
        case 16: x.scale_stride_page = 0; break;
        case 17: x.page_table = at<int32_t>(2); break;
      }
      const dustin_batch b = batch();
      EXPECT(append(&x, &x, &b), want);
      if (what == 10) continue;
      EXPECT(dense(&x, &x, &b), want);
      EXPECT(sparse(&x, &x, &b), want);
      const dustin_kv4 to = what < 12 ? kv4(200, 2, 128, 1 << 20) : paged4(1 << 20);
      EXPECT(dustin_kv4_evict(&x, nullptr, &to, nullptr, 2, at<int32_t>(), 40, 0, at<int32_t>(), 1, 40, nullptr, 0, 0, 0,
                              nullptr, 0, 0, nullptr, nullptr),
             want);
    }
    b2 = batch(0);
    EXPECT(append(&k, &v, &b2, nullptr, nullptr), DUSTIN_OK);
    b2 = batch(2, 100, 0);
    EXPECT(append(&k, &v, &b2, nullptr, nullptr), DUSTIN_OK);
    EXPECT(append(&k, nullptr, &b2, nullptr, nullptr), BAD);
    dustin_kv4 v2 = v;
    v2.num_kv_heads = 1;
    EXPECT(append(&k, &v2, &bt), BAD);
    EXPECT(append(&k, &p, &bt), BAD);  // K contiguous, V paged
  }
  {  // ---- attention
    const dustin_batch bt = batch();
    const dustin_kv4 k = kv4(), v = kv4(200, 2, 128, 1 << 20), p = paged4();
    EXPECT(sparse(&k, &v, &bt), PASSED);
    EXPECT(dense(&k, &v, &bt), PASSED);
    EXPECT(sparse(&p, &p, &bt), PASSED);
    EXPECT(sparse(&k, &v, &bt, 7), BAD);
    EXPECT(sparse(&k, &v, &bt, 8, nullptr), BAD);
    EXPECT(sparse(&k, &v, &bt, 8, fake(2)), BAD);
    EXPECT(sparse(&k, &v, &bt, 8, fake(), nullptr), BAD);
    EXPECT(sparse(&k, &v, &bt, 8, fake(), fake(4)), BAD);
    EXPECT(sparse(&k, &v, &bt, 8, fake(), fake(), nullptr), BAD);
    EXPECT(sparse(&k, &v, &bt, 8, fake(), fake(), at<int32_t>(), nullptr), BAD);
    EXPECT(sparse(&k, &v, &bt, 8, fake(), fake(), at<int32_t>(1)), BAD);
    EXPECT(sparse(&k, &v, &bt, 8, fake(), fake(), at<int32_t>(), at<int32_t>(), 3), BAD);
    EXPECT(sparse(&k, &v, &bt, 8, fake(), fake(), at<int32_t>(), at<int32_t>(), 2), PASSED);
    EXPECT(sparse(&k, &v, &bt, 8, fake(), fake(), at<int32_t>(), at<int32_t>(), 1, NAN), BAD);
    EXPECT(sparse(&k, &v, &bt, 8, fake(), fake(), at<int32_t>(), at<int32_t>(), 1, 0.f), BAD);
    EXPECT(sparse(&k, &v, &bt, 8, fake(), fake(), at<int32_t>(), at<int32_t>(), 1, 0.1f, nullptr), DUSTIN_ERR_WORKSPACE);
    EXPECT(sparse(&k, &v, &bt, 8, fake(), fake(), at<int32_t>(), at<int32_t>(), 1, 0.1f, fake(16)), DUSTIN_ERR_WORKSPACE);
    EXPECT(sparse(&k, &v, &bt, 8, fake(), fake(), at<int32_t>(), at<int32_t>(), 1, 0.1f, fake(), 256),
           DUSTIN_ERR_WORKSPACE);
    EXPECT(sparse(&k, &v, &bt, 8, fake(), fake(), at<int32_t>(), at<int32_t>(), 1, 0.1f, fake(), (size_t)1 << 40, 4), BAD);
    EXPECT(sparse(&k, &v, &bt, 8, fake(), fake(), at<int32_t>(), at<int32_t>(), 1, 0.1f, fake(), (size_t)1 << 40, 4096, -1),
           BAD);
    EXPECT(dense(&k, &v, &bt, 8, nullptr), DUSTIN_ERR_WORKSPACE);
    EXPECT(dense(&k, &v, &bt, 8, fake(), (size_t)1 << 40, -1.f), BAD);
    dustin_kv4 big_rows = kv4();
    const dustin_kv4 k64 = kv4(200, 2, 64);
    EXPECT(dense(&k64, &k64, &bt), UNSUP);
    dustin_batch b2 = batch(2, 100, 33);  // 33 x 4 rows of a head
    EXPECT(dense(&k, &v, &b2), UNSUP);
    b2 = batch(2, 100, 32);
    EXPECT(dense(&k, &v, &b2), PASSED);
    EXPECT(dustin::last_rt, 8);
    b2 = batch(1, INT32_MAX - 4096, 32);
    big_rows.capacity = INT32_MAX;
    EXPECT(dense(&big_rows, &big_rows, &b2), PASSED);
    EXPECT(dustin::last_units, 256);
    b2 = batch(40000, 100, 4);  // 80000 pairs
    EXPECT(dense(&k, &v, &b2), UNSUP);
    dustin_kv4 big = kv4();
    big.capacity = INT32_MAX;
    b2 = batch(1, INT32_MAX - 4096, 4);
    EXPECT(dense(&big, &big, &b2), PASSED);
    EXPECT(dustin::last_units, 512);  // two workgroups to a CU
    b2 = batch(1, INT32_MAX - 4095, 4);
    EXPECT(dense(&big, &big, &b2), UNSUP);
    b2 = batch(2, 100, 4, INT32_MAX - 4095);
    EXPECT(sparse(&k, &v, &b2), UNSUP);
    b2 = batch(32768, INT32_MAX - 4096, 4);  // more granules than 2^30
    EXPECT(dense(&big, &big, &b2), UNSUP);
    dustin_kv4 wide = kv4();
    wide.stride_n = ((int64_t)1 << 32);
    EXPECT(dense(&wide, &wide, &bt), UNSUP);
    b2 = batch(0);
    EXPECT(dense(&k, &v, &b2), DUSTIN_OK);
    b2 = batch(2, 100, 0);
    EXPECT(dense(&k, &v, &b2), DUSTIN_OK);
    EXPECT(sparse(&k, &v, &b2, 8, nullptr, nullptr, nullptr, nullptr), DUSTIN_OK);
    b2 = batch(2, 100, 4, 0);
    EXPECT(sparse(&k, &v, &b2, 8, fake(), fake(), nullptr), PASSED);
    EXPECT(sparse(&k, &v, &b2, 8, fake(), fake(), nullptr, nullptr), BAD);
    // the workspace that the size asks for is enough, and no byte less
    for (const int B : {1, 2, 16, 300})
      for (const int nq : {1, 4, 32})
        for (const int n : {0, 1, 100, 196 - nq}) {
          const size_t need = dustin_attn_kv4_workspace(B, 8, 2, nq, n);
          const dustin_batch b = batch(B, n, nq, n);
          EXPECT(dense(&k, &v, &b, 8, fake(), need), PASSED);
          EXPECT(dense(&k, &v, &b, 8, fake(), need - 1), DUSTIN_ERR_WORKSPACE);
        }
    EXPECT(dustin_attn_kv4_workspace(0, 8, 2, 4, 10), 0);
    EXPECT(dustin_attn_kv4_workspace(1, 7, 2, 4, 10), 0);
    EXPECT(dustin_attn_kv4_workspace(1, 8, 2, 4, -1), 0);
    EXPECT(dustin_attn_kv4_workspace(INT32_MAX, 8, 2, INT32_MAX, INT32_MAX) == 0, 0);
  }
  {  // ---- eviction
    const int32_t *idx = at<int32_t>(), *cnt = at<int32_t>();
    const dustin_kv k = kv16(), v = kv16(1 << 20), ko = kv16(2 << 20), vo = kv16(3 << 20);
    auto evict = [&](const dustin_kv* a, const dustin_kv* b, const dustin_kv* c, const dustin_kv* d, int B = 2, int G = 1,
                     int k_max = 40, const int32_t* i = at<int32_t>(), const int32_t* n = at<int32_t>(),
                     const float* w = nullptr, float* wo = nullptr, int w_len = 0, int32_t* lens = nullptr,
                     int64_t w_sb = 200) {
      return (int)dustin_kv_evict(a, b, c, d, B, i, 40, 40, n, G, k_max, w, w_sb, 0, w_len, wo, 40, 0, lens, nullptr);
    };
    EXPECT(evict(&k, &v, &ko, &vo), PASSED);
    EXPECT(evict(&k, &v, &k, &v), PASSED);
    EXPECT(evict(&k, nullptr, &ko, nullptr), PASSED);
    EXPECT(evict(&k, nullptr, &k, nullptr), PASSED);
    EXPECT(evict(&k, &v, &ko, &vo, 2, 2), PASSED);
    EXPECT(evict(&k, &v, &ko, &vo, 0), DUSTIN_OK);
    EXPECT(evict(&k, &v, &ko, &vo, 0, 1, 40, nullptr, nullptr), DUSTIN_OK);
    EXPECT(evict(&k, &v, &ko, &vo, 2, 1, 0, nullptr), PASSED);
    EXPECT(evict(&k, &v, &ko, &vo, 2, 1, 0, nullptr, nullptr), BAD);
    EXPECT(dustin_kv_evict(&k, &v, &ko, &vo, 2, idx, 40, 40, cnt, 1, 40, at<float>(), 0, 0, 200, at<float>(4096), 0, 0,
                           nullptr, nullptr),
           BAD);  // one row of weights out for two sequences
    EXPECT(dustin_kv_evict(&k, &v, &ko, &vo, 2, idx, 40, 40, cnt, 2, 40, at<float>(), 200, 0, 200, at<float>(4096), 80, 0,
                           nullptr, nullptr),
           BAD);
    EXPECT(dustin_kv_evict(&k, &v, &ko, &vo, 2, idx, 40, 40, cnt, 2, 40, at<float>(), 200, 0, 200, at<float>(4096), 80, 40,
                           nullptr, nullptr),
           PASSED);
    EXPECT(evict(nullptr, &v, &ko, &vo), BAD);
    EXPECT(evict(&k, &v, nullptr, &vo), BAD);
    EXPECT(evict(&k, &v, &ko, nullptr), BAD);
    EXPECT(evict(&k, nullptr, &ko, &vo), BAD);
    EXPECT(evict(&k, &k, &ko, &vo), BAD);
    EXPECT(evict(&k, &v, &ko, &ko), BAD);
    EXPECT(evict(&k, &v, &k, &vo), BAD);  // one of them in place
    EXPECT(evict(&k, &v, &ko, &v), BAD);
    dustin_kv odd = k;
    odd.stride_n *= 2;
    EXPECT(evict(&k, &v, &odd, &vo), BAD);  // the same memory in another layout
    EXPECT(evict(&k, &v, &ko, &vo, -1), BAD);
    EXPECT(evict(&k, &v, &ko, &vo, 2, 3), BAD);
    EXPECT(evict(&k, &v, &ko, &vo, 2, 1, -1), BAD);
    EXPECT(evict(&k, &v, &ko, &vo, 2, 1, 201), BAD);
    EXPECT(evict(&k, &v, &ko, &vo, 2, 1, 40, nullptr), BAD);
    EXPECT(evict(&k, &v, &ko, &vo, 2, 1, 40, idx, nullptr), BAD);
    EXPECT(evict(&k, &v, &ko, &vo, 2, 1, 40, at<int32_t>(1)), BAD);
    EXPECT(evict(&k, &v, &ko, &vo, 2, 1, 40, idx, cnt, at<float>()), BAD);
    EXPECT(evict(&k, &v, &ko, &vo, 2, 1, 40, idx, cnt, at<float>(), at<float>(), 0), BAD);
    EXPECT(evict(&k, &v, &ko, &vo, 2, 1, 40, idx, cnt, at<float>(2), at<float>(), 200), BAD);
    EXPECT(evict(&k, &v, &ko, &vo, 2, 1, 40, idx, cnt, at<float>(), at<float>(), 200, nullptr, -1), BAD);
    EXPECT(evict(&k, &v, &ko, &vo, 2, 1, 40, idx, cnt, at<float>(), at<float>(), 200), PASSED);
    EXPECT(evict(&k, &v, &ko, &vo, 2, 1, 40, idx, cnt, nullptr, nullptr, 0, at<int32_t>(1)), BAD);
    const dustin_kv d64 = kv16(0, 64), d96 = kv16(0, 96);
    EXPECT(evict(&d64, nullptr, &ko, nullptr), BAD);
    EXPECT(evict(&d96, nullptr, &d96, nullptr), UNSUP);
    dustin_kv one = kv16();
    one.num_kv_heads = 1;
    EXPECT(evict(&one, nullptr, &ko, nullptr), BAD);
    const dustin_kv4 k4 = kv4(), v4 = kv4(200, 2, 128, 1 << 20), p4 = paged4(2 << 20), q4 = paged4(3 << 20);
    auto evict4 = [&](const dustin_kv4* a, const dustin_kv4* b, const dustin_kv4* c, const dustin_kv4* d) {
      return (int)dustin_kv4_evict(a, b, c, d, 2, idx, 40, 40, cnt, 1, 40, nullptr, 0, 0, 0, nullptr, 0, 0, nullptr, nullptr);
    };
    EXPECT(evict4(&k4, &v4, &p4, &q4), PASSED);
    EXPECT(evict4(&p4, &q4, &p4, &q4), PASSED);
    EXPECT(evict4(&p4, &q4, &k4, &v4), PASSED);
    EXPECT(evict4(&k4, &k4, &p4, &q4), BAD);
    EXPECT(evict4(&k4, &q4, &k4, &q4), BAD);  // K contiguous, V paged
  }
  {  // ---- sampling
    const dustin_sampling s = settings();
    EXPECT(draw(&s), PASSED);
    EXPECT(draw(&s, DUSTIN_F32), PASSED);
    EXPECT(draw(&s, 2), BAD);
    EXPECT(draw(nullptr), BAD);
    EXPECT(draw(&s, DUSTIN_BF16, -1), BAD);
    EXPECT(draw(&s, DUSTIN_BF16, 0), DUSTIN_OK);
    EXPECT(draw(&s, DUSTIN_BF16, 0, 1000, nullptr, nullptr, nullptr), DUSTIN_OK);
    EXPECT(draw(&s, DUSTIN_BF16, 2, 0), BAD);
    EXPECT(draw(&s, DUSTIN_BF16, 2, (1 << 18) + 1), UNSUP);
    EXPECT(draw(&s, DUSTIN_BF16, 2, 1 << 18), PASSED);
    EXPECT(draw(&s, DUSTIN_BF16, 65536), UNSUP);
    EXPECT(draw(&s, DUSTIN_BF16, 65535, 8), PASSED);
    EXPECT(draw(&s, DUSTIN_BF16, 2, 1000, nullptr), BAD);
    EXPECT(draw(&s, DUSTIN_BF16, 2, 1000, fake(1)), BAD);
    EXPECT(draw(&s, DUSTIN_BF16, 2, 1000, fake(2)), PASSED);
    EXPECT(draw(&s, DUSTIN_F32, 2, 1000, fake(2)), BAD);
    EXPECT(draw(&s, DUSTIN_BF16, 2, 1000, fake(), nullptr), BAD);
    EXPECT(draw(&s, DUSTIN_BF16, 2, 1000, fake(), at<float>(2)), BAD);
    EXPECT(draw(&s, DUSTIN_BF16, 2, 1000, fake(), at<float>(), nullptr), BAD);
    EXPECT(draw(&s, DUSTIN_BF16, 2, 1000, fake(), at<float>(), at<int32_t>(), at<float>(1)), BAD);
    EXPECT(draw(&s, DUSTIN_BF16, 2, 1000, fake(), at<float>(), at<int32_t>(), at<float>(), 999), BAD);
    EXPECT(draw(&s, DUSTIN_BF16, 1, 1000, fake(), at<float>(), at<int32_t>(), at<float>(), 0), PASSED);
    EXPECT(draw(&s, DUSTIN_BF16, 2, 1000, fake(), at<float>(), at<int32_t>(), nullptr, 0, nullptr), DUSTIN_ERR_WORKSPACE);
    EXPECT(draw(&s, DUSTIN_BF16, 2, 1000, fake(), at<float>(), at<int32_t>(), nullptr, 0, fake(16)), DUSTIN_ERR_WORKSPACE);
    EXPECT(draw(&s, DUSTIN_BF16, 2, 1000, fake(), at<float>(), at<int32_t>(), nullptr, 0, fake(), (size_t)1 << 40, -1), BAD);
    for (int what = 0; what < 7; ++what) {
      dustin_sampling x = settings();
      switch (what) {
        case 0: x.temperature = NAN; break;
        case 1: x.top_p = NAN; break;
        case 2: x.min_p = NAN; break;
        case 3: x.temperature_b = at<float>(2); break;
        case 4: x.top_k_b = at<int32_t>(1); break;
        case 5: x.top_p_b = at<float>(3); break;
        case 6: x.min_p_b = at<float>(2); break;
      }
      EXPECT(draw(&x), BAD);
      EXPECT(verify(&x), BAD);
    }
    for (const int dtype : {DUSTIN_BF16, DUSTIN_F32})
      for (const int B : {1, 7, 512, 65535})
        for (const int V : {1, 9, 4097, 1 << 18}) {
          const size_t need = dustin_sample_workspace(B, 1, V, dtype);
          EXPECT(draw(&s, dtype, B, V, fake(), at<float>(), at<int32_t>(), nullptr, 0, fake(), need), PASSED);
          EXPECT(draw(&s, dtype, B, V, fake(), at<float>(), at<int32_t>(), nullptr, 0, fake(), need - 1),
                 DUSTIN_ERR_WORKSPACE);
        }
    EXPECT(dustin_sample_workspace(0, 1, 100, DUSTIN_BF16), 0);
    EXPECT(dustin_sample_workspace(1, 1, 100, 5), 0);
    EXPECT(dustin_sample_workspace(65535, 2, 100, DUSTIN_BF16), 0);
    // ---- verification
    EXPECT(verify(&s), PASSED);
    EXPECT(verify(&s, 1, nullptr, nullptr), PASSED);
    EXPECT(verify(&s, 64), PASSED);
    EXPECT(verify(&s, 65), UNSUP);
    EXPECT(verify(&s, 0), BAD);
    EXPECT(verify(&s, -1), BAD);
    EXPECT(verify(&s, 5, nullptr), BAD);
    EXPECT(verify(&s, 5, at<int32_t>(2)), BAD);
    EXPECT(verify(&s, 5, at<int32_t>(), nullptr), BAD);
    EXPECT(verify(&s, 5, at<int32_t>(), at<float>(), nullptr), BAD);
    EXPECT(verify(&s, 5, at<int32_t>(), at<float>(), at<int32_t>(), nullptr), BAD);
    EXPECT(verify(&s, 5, at<int32_t>(), at<float>(), at<int32_t>(), at<int32_t>(), at<float>(2)), BAD);
    EXPECT(verify(&s, 5, at<int32_t>(), at<float>(), at<int32_t>(), at<int32_t>(), at<float>()), PASSED);
    EXPECT(verify(&s, 5, at<int32_t>(), at<float>(), at<int32_t>(), at<int32_t>(), nullptr, at<int32_t>(2)), BAD);
    EXPECT(verify(&s, 5, at<int32_t>(), at<float>(), at<int32_t>(), at<int32_t>(), nullptr, nullptr, 0), DUSTIN_OK);
    EXPECT(verify(&s, 5, at<int32_t>(), at<float>(), at<int32_t>(), at<int32_t>(), nullptr, nullptr, 20000), UNSUP);
    EXPECT(verify(&s, 5, at<int32_t>(), at<float>(), at<int32_t>(), at<int32_t>(), nullptr, nullptr, 2, 64),
           DUSTIN_ERR_WORKSPACE);
    EXPECT(verify(&s, 5, at<int32_t>(), at<float>(), at<int32_t>(), at<int32_t>(), nullptr, nullptr, 2, (size_t)1 << 40,
                  1000, -1),
           BAD);
    for (const int B : {1, 33}) {
      const size_t need = dustin_sample_workspace(B, 5, 5003, DUSTIN_F32);
      EXPECT(verify(&s, 5, at<int32_t>(), at<float>(), at<int32_t>(), at<int32_t>(), nullptr, nullptr, B, need, 5003), PASSED);
      EXPECT(verify(&s, 5, at<int32_t>(), at<float>(), at<int32_t>(), at<int32_t>(), nullptr, nullptr, B, need - 1, 5003),
             DUSTIN_ERR_WORKSPACE);
    }
  }
  printf("%s: %d failed expectations\n", failures ? "FAILED" : "ok", failures);
  return failures ? 1 : 0;
}
