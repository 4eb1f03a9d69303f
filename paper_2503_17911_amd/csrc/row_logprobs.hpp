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
