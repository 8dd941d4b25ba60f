// sample.hpp -- argument blocks of the sampling kernels (internal).
#pragma once

#include "kernels.hpp"

namespace dustin {

// Tokens are ranked by (logit descending, index ascending) through one number, smaller for the better: the logit's
// order-preserving key, complemented, over the index.
constexpr int kSampleIdxBits = 18;
constexpr int kSampleMaxVocab = 1 << kSampleIdxBits;

// A token's weight, 2^((x - top) log2(e) / T) of the row's largest logit, is summed as a multiple of 2^-44: sums of
// integers do not depend on their order, 2^18 tokens stay below 2^62, and a weight is off by at most 2^-45.  Weights
// below 2^-45, half a unit, count as zero.
constexpr int kSampleFrac = 44;
constexpr int kSampleBins = 368;     // eighths of octaves from the largest weight down to 2^-46
constexpr int kSampleFew = 1024;     // tokens of a list that holds all that may be kept
constexpr int kSampleList = 4096;    // tokens of a list
constexpr int kSampleMaxWindow = 64; // tokens of a verification window
constexpr int kSamplePieces = 1024;  // 16-byte pieces of a chunk of a row (with 512, 128 rows took 90 us for 72, one 24)
constexpr int kSampleMaxChunks = 65;  // 2^18 fp32 logits, wherever the row begins

struct SampleRow {  // what is known of a row once its filters are resolved
  uint64_t last;    // rank of the last kept token (0: none is)
  uint64_t sum;     // of the kept weights
  float top;        // largest logit
};

// How the rest of a row is done, from its histogram.
enum SampleMode : int32_t {
  kRowWhole = 1,  // every token is kept
  kRowFew = 2,    // all that may be kept are few: ranks lo .. hi
  kRowList = 3,   // the last kept token's eighth of an octave is ranks lo .. hi
  kRowRead = 4,   // read the row as often as it takes
};
struct SamplePlan {
  int32_t mode, bin;
  uint64_t lo, hi;          // ranks of the tokens to list
  uint64_t before_cnt, before_sum;  // kRowList: tokens of better eighths
  uint64_t all_sum;
  uint64_t least;           // rank of the last token that min_p keeps (~0: of any)
  double target;            // kRowList: running count or sum at which the last token is reached (negative: at `least`)
  int32_t by_count;
};

struct SampleArgs {
  const void* logits;
  int64_t sb, st;  // strides of sequences and of a sequence's rows, in elements
  int32_t batch, rows_per_seq, vocab;
  const int32_t* n_query;  // rows of a sequence, or NULL (= rows_per_seq)
  const float* temperature;
  const int32_t* top_k;
  const float* top_p;
  const float* min_p;  // [batch] or NULL: the scalars
  float s_temperature, s_top_p, s_min_p;
  int32_t s_top_k;
  const float* u;  // [batch]
  int32_t* token;  // [batch]
  float* probs;    // sampling: [batch][vocab] or NULL
  int64_t probs_sb;
  // verification
  const int32_t* draft;
  int64_t draft_sb;
  const float* q;  // or NULL: the drafts were certain
  int64_t q_sb, q_st;
  const float* u_accept;
  int64_t ua_sb;
  int32_t* accepted;
  // chunks of a row, and what is kept of them
  int32_t chunks;
  float* c_top;       // [rows][chunks] largest logit
  uint64_t* c_best;   // best rank
  uint64_t* c_sum;    // sum of weights, against the chunk's largest
  uint64_t* h_sum;    // [rows][chunks][kSampleBins]
  uint32_t* h_cnt;
  SampleRow* row;     // [rows]
  uint64_t* list;     // [rows][kSampleList] ranks
  int32_t parts;      // workgroups that list a row's tokens
  uint64_t* r_sum;    // [batch][chunks][2]: sums of what is left of the distribution, and of it whole
  uint32_t* arrived;  // [rows], zero between calls
  uint32_t* listed;   // [rows], zero between calls
};

hipError_t launch_sample(const SampleArgs& a, bool bf16, hipStream_t stream);
hipError_t launch_verify_sample(const SampleArgs& a, bool bf16, hipStream_t stream);

}  // namespace dustin
