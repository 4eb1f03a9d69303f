// What the two directions of the rows' log probabilities share.
#pragma once
#include "tile_product.hpp"

namespace ann {

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.693147180559945309417f;

// A launch has fewer than 2^32 lanes: 256 to a query, two to a row.
constexpr uint64_t kMaxRows = (1ull << 31) - 256;
constexpr uint32_t kMaxQueries = 1u << 24;

// s[i][j] = scale <q_i, rows_j> + bias_j
struct ScoreTable {
  const void *q, *rows;
  const float *bias;
  uint64_t q_stride, row_stride;
  uint32_t nq, n, d;
  float scale;
};

inline ScoreTable score_table(const ann_row_scores &s) {
  return {s.q, s.rows, s.row_bias, s.q_stride, s.row_stride, s.nq, (uint32_t)s.n, s.d, s.scale};
}

// What the gradients of the scores are asked for.  With `every`, g_logprob is a weight of every query's probabilities, whether a row is given
// or not (targets, g_entropy: NULL), G of 16-bit rows is multiplied in two parts of 16 bits, and what more there is to single elements of it is added in fp32:
//   more_part    to dq: another part of its sums, which is in the workspace already (times what G is multiplied by)
//   slots        to drows[j] (and drow_bias[j], its column d): sums[slots[j]] of more_ld elements, where slots[j] is not ANN_PAD_ID
struct GradArgs {
  ScoreTable g;
  const uint32_t *targets;
  const float *lse, *entropy, *g_logprob, *g_entropy;
  const float *scaling;  // [2]: what G is multiplied by before it is rounded, and its inverse (f16)
  float *rest;           // [nq]: what the rounding of the given row's element left (16 bits)
  bool every, more_part;
  const uint32_t *slots;
  const float *sums;
  uint32_t more_ld;
};

struct GradOut {
  void *dq, *drows;
  float *drow_bias;
  uint64_t dq_stride, drows_stride;
};

constexpr uint32_t kFewGradQueries = 256;  // up to so many, the rows' gradient takes all of G's remainders

uint64_t scores_backward_bytes(uint32_t nq, uint64_t n, uint32_t d, uint32_t type, bool more);
float *scores_backward_more_part(uint32_t nq, uint64_t n, uint32_t d, uint32_t type, void *workspace);  // [nq][d]; there are queries and rows
// scaling: of f16, [2]; written by launch_grad_scaling.
ann_status launch_grad_scaling(const GradArgs &a, float *scaling, hipStream_t st);
// a.scaling of f16: NULL to have it found (in the workspace).
ann_status scores_backward(uint32_t type, const GradArgs &a, const GradOut &o, void *workspace, hipStream_t st);

// lse (and logprob: 0) as ann_row_logprobs without targets and alternatives, in a workspace of its size; wide_lse: lse before it is rounded.  fp32 scores
// are as exact as their gradients': what is taken off lse, a given row's score, is exact, and where that row has nearly all probability their difference is
// what the scores err by.
ann_status row_statistics(const ann_row_scores &s, float *logprob, float *lse, double *wide_lse, void *workspace, hipStream_t st);

ann_status check_scores(const char *what, const ann_row_scores *s);
ann_status check_workspace(const char *what, const void *workspace, uint64_t bytes, uint64_t need);

// Hands out parts of a workspace, each aligned to 256 bytes.
struct Parts {
  uint64_t bytes = 0;
  uint64_t take(uint64_t size) {
    const uint64_t at = bytes;
    bytes += (size + 255) / 256 * 256;
    return at;
  }
};

}  // namespace ann
