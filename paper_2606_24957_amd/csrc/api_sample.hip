// api_sample.hip -- the extern "C" boundary of sampling and of the verification of drafted tokens: argument validation,
// workspace layout, launch configuration.  Validation happens before any HIP call.
#include <math.h>

#include "sample.hpp"
#include "validate.hpp"

using namespace dustin;

namespace {

constexpr int kMaxRows = 65535;  // rows of logits of a call: a dimension of the launch

constexpr size_t kCounters = (kMaxRows + 1) * sizeof(uint32_t);  // of each kind

// The workspace begins with the arrival and list counters, whatever a call's sizes are.
struct SampleWs {
  int chunks;
  size_t row, list, c_top, c_best, c_sum, r_sum, h_cnt, h_sum, total;
};

SampleWs sample_ws(int64_t batch, int64_t rows, int64_t vocab, bool bf16) {
  SampleWs w;
  const int64_t pieces = vocab / (bf16 ? 8 : 4) + 2;  // a row may begin and end inside one
  w.chunks = (int)((pieces + kSamplePieces - 1) / kSamplePieces);
  size_t at = 2 * kCounters;
  auto take = [&](size_t bytes) {
    const size_t x = at;
    at += round_up(bytes, kAlign);
    return x;
  };
  const size_t n = (size_t)rows * w.chunks;
  w.row = take((size_t)rows * sizeof(SampleRow));
  w.list = take((size_t)rows * kSampleList * sizeof(uint64_t));
  w.c_top = take(n * sizeof(float));
  w.c_best = take(n * sizeof(uint64_t));
  w.c_sum = take(n * sizeof(uint64_t));
  w.r_sum = take((size_t)batch * w.chunks * 2 * sizeof(uint64_t));
  w.h_cnt = take(n * kSampleBins * sizeof(uint32_t));
  w.h_sum = take(n * kSampleBins * sizeof(uint64_t));
  w.total = at;
  return w;
}

dustin_status common(SampleArgs& a, const void* logits, int32_t dtype, int64_t sb, int64_t st, int32_t batch,
                     int32_t nq_max, int32_t vocab, const dustin_sampling* set, const float* u, int32_t* token) {
  if ((batch > 0 && (!logits || !u || !token)) || !set || batch < 0 || nq_max < 0 || vocab <= 0 || sb < 0 || st < 0)
    return DUSTIN_ERR_INVALID_ARG;
  if (dtype != DUSTIN_BF16 && dtype != DUSTIN_F32) return DUSTIN_ERR_INVALID_ARG;
  if (!aligned(logits, dtype == DUSTIN_BF16 ? 2 : 4) || !aligned(u, 4) || !aligned(token, 4) ||
      !aligned(set->temperature_b, 4) || !aligned(set->top_k_b, 4) || !aligned(set->top_p_b, 4) ||
      !aligned(set->min_p_b, 4))
    return DUSTIN_ERR_INVALID_ARG;
  if ((!set->temperature_b && isnan(set->temperature)) || (!set->top_p_b && isnan(set->top_p)) ||
      (!set->min_p_b && isnan(set->min_p)))
    return DUSTIN_ERR_INVALID_ARG;
  if (vocab > kSampleMaxVocab || (int64_t)batch * (nq_max > 0 ? nq_max : 1) > kMaxRows) return DUSTIN_ERR_UNSUPPORTED;
  memset(&a, 0, sizeof a);
  a.logits = logits;
  a.sb = sb;
  a.st = st;
  a.batch = batch;
  a.rows_per_seq = nq_max;
  a.vocab = vocab;
  a.temperature = set->temperature_b;
  a.top_k = set->top_k_b;
  a.top_p = set->top_p_b;
  a.min_p = set->min_p_b;
  a.s_temperature = set->temperature;
  a.s_top_k = set->top_k;
  a.s_top_p = set->top_p;
  a.s_min_p = set->min_p;
  a.u = u;
  a.token = token;
  return DUSTIN_OK;
}

dustin_status place(SampleArgs& a, bool bf16, void* ws, size_t ws_bytes) {
  const SampleWs w = sample_ws(a.batch, (int64_t)a.batch * a.rows_per_seq, a.vocab, bf16);
  if (!ws || ws_bytes < w.total || !aligned(ws, kAlign)) return DUSTIN_ERR_WORKSPACE;
  char* base = static_cast<char*>(ws);
  a.chunks = w.chunks;
  a.arrived = reinterpret_cast<uint32_t*>(base);
  a.listed = reinterpret_cast<uint32_t*>(base + kCounters);
  const int64_t rows = (int64_t)a.batch * a.rows_per_seq;
  a.parts = (int32_t)(rows >= 256 ? 1 : 256 / rows);  // (one workgroup to a CU)
  if (a.parts > w.chunks) a.parts = w.chunks;
  a.list = reinterpret_cast<uint64_t*>(base + w.list);
  a.row = reinterpret_cast<SampleRow*>(base + w.row);
  a.c_top = reinterpret_cast<float*>(base + w.c_top);
  a.c_best = reinterpret_cast<uint64_t*>(base + w.c_best);
  a.c_sum = reinterpret_cast<uint64_t*>(base + w.c_sum);
  a.r_sum = reinterpret_cast<uint64_t*>(base + w.r_sum);
  a.h_cnt = reinterpret_cast<uint32_t*>(base + w.h_cnt);
  a.h_sum = reinterpret_cast<uint64_t*>(base + w.h_sum);
  return DUSTIN_OK;
}

}  // namespace

extern "C" {

size_t dustin_sample_workspace(int32_t batch, int32_t nq_max, int32_t vocab, int32_t dtype) {
  if (batch <= 0 || nq_max <= 0 || vocab <= 0 || vocab > kSampleMaxVocab || (int64_t)batch * nq_max > kMaxRows ||
      (dtype != DUSTIN_BF16 && dtype != DUSTIN_F32))
    return 0;
  return sample_ws(batch, (int64_t)batch * nq_max, vocab, dtype == DUSTIN_BF16).total;
}

dustin_status dustin_sample(const void* logits, int32_t dtype, int64_t l_sb, int32_t batch, int32_t vocab,
                            const dustin_sampling* set, const float* u, int32_t* token, float* probs, int64_t probs_sb,
                            void* workspace, size_t workspace_bytes, void* stream) {
  SampleArgs a;
  dustin_status st = common(a, logits, dtype, l_sb, 0, batch, 1, vocab, set, u, token);
  if (st != DUSTIN_OK) return st;
  if (probs && (!aligned(probs, 4) || (batch > 1 && probs_sb < vocab))) return DUSTIN_ERR_INVALID_ARG;
  if (batch == 0) return DUSTIN_OK;
  st = place(a, dtype == DUSTIN_BF16, workspace, workspace_bytes);
  if (st != DUSTIN_OK) return st;
  a.probs = probs;
  a.probs_sb = probs_sb;
  return launch_sample(a, dtype == DUSTIN_BF16, static_cast<hipStream_t>(stream)) == hipSuccess ? DUSTIN_OK
                                                                                               : DUSTIN_ERR_LAUNCH;
}

dustin_status dustin_verify_sample(const void* logits, int32_t dtype, int64_t l_sb, int64_t l_st, int32_t batch,
                                   int32_t nq_max, const int32_t* n_query, int32_t vocab, const dustin_sampling* set,
                                   const int32_t* draft, int64_t draft_sb, const float* draft_probs, int64_t q_sb,
                                   int64_t q_st, const float* u_accept, int64_t ua_sb, const float* u,
                                   int32_t* accepted, int32_t* token, void* workspace, size_t workspace_bytes,
                                   void* stream) {
  SampleArgs a;
  dustin_status st = common(a, logits, dtype, l_sb, l_st, batch, nq_max, vocab, set, u, token);
  if (st != DUSTIN_OK) return st;
  if ((batch > 0 && !accepted) || !aligned(accepted, 4) || !aligned(n_query, 4) || nq_max < 1) return DUSTIN_ERR_INVALID_ARG;
  if (nq_max > kSampleMaxWindow) return DUSTIN_ERR_UNSUPPORTED;
  if (nq_max > 1 && ((batch > 0 && (!draft || !u_accept)) || !aligned(draft, 4) || !aligned(u_accept, 4) || draft_sb < 0 || ua_sb < 0))
    return DUSTIN_ERR_INVALID_ARG;
  if (draft_probs && (!aligned(draft_probs, 4) || q_sb < 0 || q_st < 0)) return DUSTIN_ERR_INVALID_ARG;
  if (batch == 0) return DUSTIN_OK;
  st = place(a, dtype == DUSTIN_BF16, workspace, workspace_bytes);
  if (st != DUSTIN_OK) return st;
  a.n_query = n_query;
  a.draft = draft;
  a.draft_sb = draft_sb;
  a.q = draft_probs;
  a.q_sb = q_sb;
  a.q_st = q_st;
  a.u_accept = u_accept;
  a.ua_sb = ua_sb;
  a.accepted = accepted;
  return launch_verify_sample(a, dtype == DUSTIN_BF16, static_cast<hipStream_t>(stream)) == hipSuccess
             ? DUSTIN_OK
             : DUSTIN_ERR_LAUNCH;
}

}  // extern "C"
