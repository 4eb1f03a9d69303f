// Entries in the order of their ids, equal ids in the order of their positions: what gradients of rows that are named by ids are summed by.
#pragma once
#include "ann_internal.hpp"

namespace ann {

constexpr uint32_t kSmallSort = 4096;  // up to so many ids are sorted by one workgroup

// A plan for `n` ids of which those below `rows` count; the others come last, as the id `rows`.
struct IdSortPlan {
  uint32_t n = 0, rows = 0, passes = 0, bits = 0, blocks = 0, rounds = 0;  // bits: of a pass' digit; rounds: of kSortThreads entries to a block
  uint64_t bytes = 0, keys_at[2] = {}, at_at[2] = {}, counts_at = 0, totals_at = 0;
};
IdSortPlan id_sort_plan(uint64_t n, uint64_t rows);  // n < 2^31, rows <= 2^31

// keys[i], positions[i]: the i-th entry's id and its place among the ids given.  hit (NULL allowed, and with up to kSmallSort ids): one bit to a
// row, set for the rows that an id names ((rows + 31) / 32 words, cleared here first).  `workspace` holds plan.bytes; the results are in it.
struct SortedIds {
  const uint32_t *keys, *positions;
};
ann_status sort_ids(const IdSortPlan &plan, const uint32_t *ids, void *workspace, uint32_t *hit, hipStream_t st, SortedIds &out);

}  // namespace ann
