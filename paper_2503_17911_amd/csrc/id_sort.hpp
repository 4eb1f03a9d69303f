// Entries in the order of their ids, equal ids in the order of their positions: what gradients of rows that are named by ids are summed by.
//
// A stable radix sort of ids with their positions, from the lowest digit up: one to three passes of up to 11 bits.
//
// A pass counts the digits of every block's entries, then every block places its entries behind the smaller digits' and the earlier blocks'.
// The place within a block follows the entries' order (a wavefront finds the lanes with its digit by one ballot to a bit, and counts
// rounds and wavefronts one after the other), so equal ids stay in the order of their positions and the result does not depend on
// timing.  With few blocks a block adds up the counts of the others itself; with many a kernel between the two does.  Up to kSmallSort entries
// are put in order by one kernel that compares all with all.  Bound by launches and the counters' latency: 80,000 ids are 320 KB and take
// two passes of 5 + 9 us.
// Work that does not wait for the order may run beside it, in workgroups of the same launches.
#pragma once
#include "ann_internal.hpp"
#include "device_utils.hpp"

namespace ann {

constexpr uint32_t kSmallSort = 12288;  // up to so many ids are put in order by counting (16,000: 33 us, 32 by two passes; 8,290: 16)

// A plan for `n` ids of which those below `rows` count; the others come last, as the id `rows`.
struct IdSortPlan {
  uint32_t n = 0, rows = 0, passes = 0, bits = 0, blocks = 0, rounds = 0;  // bits: of a pass' digit; rounds: of kSortThreads entries to a block
  uint64_t bytes = 0, keys_at[2] = {}, at_at[2] = {}, counts_at = 0, totals_at = 0;
};

// keys[i], positions[i]: the i-th entry's id and its place among the ids given; in the workspace.
struct SortedIds {
  const uint32_t *keys, *positions;
};

// hit (NULL allowed, and with up to kSmallSort ids): a byte to a row, 1 for the rows that an id names and 0 for the others
// ((rows + 3) / 4 words are written).  `workspace` holds plan.bytes.
template <typename Beside>
static ann_status sort_ids(const IdSortPlan &plan, const uint32_t *ids, void *workspace, uint8_t *hit, Beside beside, hipStream_t st, SortedIds &out);

// Work beside the sorting: operator()(stage, part, parts) is called by all lanes of workgroups of kSortThreads (kSmallThreads) lanes, in stage 0
// (up to kSmallSort ids) or in the stages 1 and 2 (more, from two passes on), when `hit` is complete.
struct NothingBeside {
  uint32_t blocks = 0;  // workgroups, in each stage
  __device__ __forceinline__ void operator()(uint32_t, uint32_t, uint32_t) const {}
};

constexpr uint32_t kSortThreads = 512, kSortWaves = kSortThreads / kWave, kSortRounds = 4;  // (80,000 ids: 35 us for both passes, 41 by eight rounds, 37 by 1,024 lanes)
constexpr uint32_t kMaxBits = 11, kMaxDigits = 1u << kMaxBits;
constexpr uint32_t kFewBlocks = 64;      // up to so many, a block adds the others' counts itself
constexpr uint32_t kMostBlocks = 4096;   // beyond, blocks take more rounds
constexpr uint32_t kSmallThreads = 1024;

inline IdSortPlan id_sort_plan(uint64_t n, uint64_t rows) {  // n < 2^31, rows <= 2^31
  IdSortPlan p;
  p.n = (uint32_t)n, p.rows = (uint32_t)rows;
  uint32_t width = 1;  // bits of ids up to `rows`
  while (width < 32 && (rows >> width) != 0) ++width;
  p.passes = n <= kSmallSort ? 1 : (width + kMaxBits - 1) / kMaxBits;
  p.bits = n <= kSmallSort ? width : (width + p.passes - 1) / p.passes;
  p.rounds = kSortRounds;
  while ((n + (uint64_t)p.rounds * kSortThreads - 1) / ((uint64_t)p.rounds * kSortThreads) > kMostBlocks) p.rounds *= 2;
  p.blocks = (uint32_t)((n + (uint64_t)p.rounds * kSortThreads - 1) / ((uint64_t)p.rounds * kSortThreads));
  const auto take = [&](uint64_t size) {
    const uint64_t at = p.bytes;
    p.bytes += (size + 255) / 256 * 256;
    return at;
  };
  for (int i = 0; i < 2; ++i) p.keys_at[i] = take(n * 4), p.at_at[i] = take(n * 4);
  if (n > kSmallSort) p.counts_at = take((uint64_t)p.blocks * (1u << p.bits) * 4), p.totals_at = take((1u << p.bits) * 4);
  return p;
}

// The sum over the lanes before this one, and `all` over all of the workgroup's.  room: a word to a wavefront and one more.
template <uint32_t THREADS>
__device__ __forceinline__ uint32_t exclusive_sum(uint32_t v, uint32_t *room, uint32_t &all) {
  const uint32_t through = (uint32_t)wave_inclusive_scan_i32((int)v);
  __syncthreads();  // (room is free)
  if (threadIdx.x % kWave == kWave - 1) room[threadIdx.x / kWave] = through;
  __syncthreads();
  uint32_t before = 0;
  all = 0;
  for (uint32_t w = 0; w < THREADS / kWave; ++w) {
    if (w < threadIdx.x / kWave) before += room[w];
    all += room[w];
  }
  return before + through - v;
}

// The lanes whose digit is `wanted` (the lane's own, mostly), of those that have one.
__device__ __forceinline__ uint64_t lanes_with(uint32_t digit, bool there, uint32_t wanted, uint32_t bits) {
  uint64_t same = __ballot(there);
  for (uint32_t b = 0; b < bits; ++b) {
    const uint64_t with = __ballot(digit >> b & 1);
    same &= wanted >> b & 1 ? with : ~with;
  }
  return same;
}

struct SortPass {
  const uint32_t *keys, *at;  // at NULL: the first pass, whose keys are the ids as given
  uint32_t *out_keys, *out_at, *counts, *totals;
  uint8_t *hit;
  uint32_t n, rows, shift, bits, rounds, blocks;
};

__device__ __forceinline__ uint32_t sort_key(const SortPass &p, uint32_t i) {
  const uint32_t key = p.keys[i];
  return !p.at && key > p.rows ? p.rows : key;
}

// counts[block][digit]
template <typename Beside>
__global__ __launch_bounds__(kSortThreads) void sort_count_kernel(SortPass p, Beside beside) {
  if (blockIdx.x >= p.blocks) return beside(1, blockIdx.x - p.blocks, gridDim.x - p.blocks);
  __shared__ uint32_t count[kMaxDigits];
  const uint32_t digits = 1u << p.bits, first = blockIdx.x * p.rounds * kSortThreads;
  for (uint32_t d = threadIdx.x; d < digits; d += kSortThreads) count[d] = 0;
  if (p.hit)
    for (uint64_t w = (uint64_t)blockIdx.x * kSortThreads + threadIdx.x; w < (p.rows + 3ull) / 4; w += (uint64_t)p.blocks * kSortThreads) ((uint32_t *)p.hit)[w] = 0;
  __syncthreads();
  for (uint32_t r0 = 0; r0 < p.rounds; r0 += kSortRounds) {
    uint32_t key[kSortRounds];
#pragma unroll
    for (uint32_t r = 0; r < kSortRounds; ++r) {
      const uint64_t i = (uint64_t)first + (r0 + r) * kSortThreads + threadIdx.x;
      key[r] = i < p.n ? sort_key(p, (uint32_t)i) : 0;
    }
#pragma unroll
    for (uint32_t r = 0; r < kSortRounds; ++r)
      if ((uint64_t)first + (r0 + r) * kSortThreads + threadIdx.x < p.n) atomicAdd(&count[key[r] >> p.shift & (digits - 1)], 1u);
  }
  __syncthreads();
  for (uint32_t d = threadIdx.x; d < digits; d += kSortThreads) p.counts[(uint64_t)blockIdx.x * digits + d] = count[d];
}

// counts[block][digit] becomes the sum over the blocks before; totals[digit] that over all.  64 digits to a workgroup, 16 runs of blocks.
template <typename Beside>
__global__ __launch_bounds__(1024) void sort_scan_kernel(SortPass p) {
  const uint32_t blocks = p.blocks;
  __shared__ uint32_t runs[16][64];
  const uint32_t digits = 1u << p.bits, lane = threadIdx.x % 64, run = threadIdx.x / 64, d = blockIdx.x * 64 + lane;
  const uint32_t begin = (uint64_t)blocks * run / 16, end = (uint64_t)blocks * (run + 1) / 16;
  uint32_t sum = 0;
  if (d < digits)
    for (uint32_t b = begin; b < end; ++b) sum += p.counts[(uint64_t)b * digits + d];
  runs[run][lane] = sum;
  __syncthreads();
  if (d >= digits) return;
  uint32_t before = 0;
  for (uint32_t r = 0; r < run; ++r) before += runs[r][lane];
  for (uint32_t b = begin; b < end; ++b) {
    const uint32_t c = p.counts[(uint64_t)b * digits + d];
    p.counts[(uint64_t)b * digits + d] = before;
    before += c;
  }
  if (run == 15) p.totals[d] = before;
}

// SCANNED: by the kernel before.
template <bool SCANNED, typename Beside>
__global__ __launch_bounds__(kSortThreads) void sort_place_kernel(SortPass p, Beside beside) {
  if (blockIdx.x >= p.blocks) return beside(2, blockIdx.x - p.blocks, gridDim.x - p.blocks);
  __shared__ uint32_t place[kMaxDigits], of_wave[kSortWaves][kMaxDigits], room[kSortWaves + 1];
  const uint32_t digits = 1u << p.bits, wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
  const uint32_t per_wave = p.rounds * kWave;
  const uint64_t first = (uint64_t)blockIdx.x * p.rounds * kSortThreads + (uint64_t)wave * per_wave;  // a wavefront's entries lie side by side
  // where each digit's entries of this block begin
  uint32_t carry = 0;
  for (uint32_t d0 = 0; d0 < digits; d0 += kSortThreads) {
    const uint32_t d = d0 + threadIdx.x;
    uint32_t total = 0, before = 0;
    if (d < digits) {
      if constexpr (SCANNED) {
        total = p.totals[d], before = p.counts[(uint64_t)blockIdx.x * digits + d];
      } else {
#pragma unroll 16
        for (uint32_t b = 0; b < p.blocks; ++b) {
          const uint32_t c = p.counts[(uint64_t)b * digits + d];
          before += b < blockIdx.x ? c : 0;
          total += c;
        }
      }
    }
    uint32_t all;
    const uint32_t smaller = exclusive_sum<kSortThreads>(total, room, all);
    if (d < digits) place[d] = carry + smaller + before;
    carry += all;
  }
  for (uint32_t d = threadIdx.x; d < digits * kSortWaves; d += kSortThreads) of_wave[d / digits][d % digits] = 0;
  __syncthreads();
  // (with kSortRounds rounds, as a rule, they are read once)
  uint32_t key[kSortRounds], at[kSortRounds];
  const auto read = [&](uint32_t r0) {
#pragma unroll
    for (uint32_t r = 0; r < kSortRounds; ++r) {
      const uint64_t i = first + (r0 + r) * kWave + lane;
      key[r] = i < p.n ? sort_key(p, (uint32_t)i) : 0, at[r] = i < p.n ? (p.at ? p.at[i] : (uint32_t)i) : 0;
    }
  };
  for (uint32_t r0 = 0; r0 < p.rounds; r0 += kSortRounds) {
    read(r0);
#pragma unroll
    for (uint32_t r = 0; r < kSortRounds; ++r)
      if (first + (r0 + r) * kWave + lane < p.n) atomicAdd(&of_wave[wave][key[r] >> p.shift & (digits - 1)], 1u);
  }
  __syncthreads();
  for (uint32_t d = threadIdx.x; d < digits; d += kSortThreads) {
    uint32_t to = place[d];
    for (uint32_t w = 0; w < kSortWaves; ++w) {
      const uint32_t c = of_wave[w][d];
      of_wave[w][d] = to;
      to += c;
    }
  }
  __syncthreads();
  for (uint32_t r0 = 0; r0 < p.rounds; r0 += kSortRounds) {
    if (p.rounds > kSortRounds) read(r0);
#pragma unroll
    for (uint32_t r = 0; r < kSortRounds; ++r) {
      const bool there = first + (r0 + r) * kWave + lane < p.n;
      const uint32_t digit = key[r] >> p.shift & (digits - 1);
      const uint64_t same = lanes_with(digit, there, digit, p.bits);
      const uint32_t rank = __popcll(same & ((1ull << lane) - 1));
      if (there) {
        const uint32_t to = of_wave[wave][digit] + rank;
        p.out_keys[to] = key[r], p.out_at[to] = at[r];
        if (p.hit && key[r] < p.rows) p.hit[key[r]] = 1;  // (whoever writes it, it is a 1; a bit to a row by atomics took 170 us where one id is frequent)
      }
      // the first of the lanes with the digit moves its place on, once all have read it
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
      if (there && rank == 0) of_wave[wave][digit] += __popcll(same);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
  }
}

// Up to kSmallSort entries: an entry's place is the number of entries before it in the order, counted against all of them (one workgroup's
// radix sort of 5,000 took 16 us, the passes of many some 27).  A workgroup takes 16 entries, the keys in LDS; 64 slices of the keys to its lanes, whose
// counts are joined in LDS.  5,000: 8 us, bound by the comparisons (n^2 of two instructions) and the reads of LDS alike.  (Two entries to a lane halve the reads
// and the workgroups: 9.2 us; keys through the scalar cache: 13.)
constexpr uint32_t kSmallOwn = 16;
template <typename Beside>
__global__ __launch_bounds__(kSmallThreads) void sort_small_kernel(SortPass p, Beside beside) {
  constexpr uint32_t kSlices = kSmallThreads / kSmallOwn;
  __shared__ __attribute__((aligned(16))) uint32_t keys[kSmallSort + 8 * kSlices];
  __shared__ uint32_t counts[kSmallOwn];
  if (blockIdx.x >= p.blocks) return beside(0, blockIdx.x - p.blocks, gridDim.x - p.blocks);
  // (pieces of 16 bytes, an odd number: slices side by side lie in other banks)
  const uint32_t slice_keys = ((p.n + kSlices - 1) / kSlices + 3) / 8 * 8 + 4, padded = slice_keys * kSlices;
  for (uint32_t i0 = threadIdx.x; i0 < padded; i0 += 8 * kSmallThreads) {  // (eight on their way)
    uint32_t k[8];
#pragma unroll
    for (uint32_t u = 0; u < 8; ++u) k[u] = i0 + u * kSmallThreads < p.n ? sort_key(p, i0 + u * kSmallThreads) : 0xFFFFFFFFu;
#pragma unroll
    for (uint32_t u = 0; u < 8; ++u)
      if (i0 + u * kSmallThreads < padded) keys[i0 + u * kSmallThreads] = k[u];
  }
  if (threadIdx.x < kSmallOwn) counts[threadIdx.x] = 0;
  __syncthreads();
  const uint32_t own = blockIdx.x * kSmallOwn + threadIdx.x % kSmallOwn, begin = threadIdx.x / kSmallOwn * slice_keys, end = begin + slice_keys;
  const uint32_t key = own < p.n ? keys[own] : 0;
  uint32_t before = 0;
  if (own < begin || own >= end) {
    const uint32_t below = key + (own >= end);  // (equal ids before it stay before it; ids are at most 2^31)
#pragma unroll 4
    for (uint32_t j = begin; j < end; j += 4) {
      const uint4 k = *(const uint4 *)(keys + j);
      before += (k.x < below) + (k.y < below) + (k.z < below) + (k.w < below);
    }
  } else {
#pragma unroll 4
    for (uint32_t j = begin; j < end; j += 4) {
      const uint4 k = *(const uint4 *)(keys + j);
      before += (k.x < key + (j < own)) + (k.y < key + (j + 1 < own)) + (k.z < key + (j + 2 < own)) + (k.w < key + (j + 3 < own));
    }
  }
  atomicAdd(&counts[threadIdx.x % kSmallOwn], before);
  __syncthreads();
  if (threadIdx.x < kSmallOwn && own < p.n) p.out_keys[counts[threadIdx.x]] = key, p.out_at[counts[threadIdx.x]] = own;
}

template <typename Beside>
static ann_status sort_ids(const IdSortPlan &plan, const uint32_t *ids, void *workspace, uint8_t *hit, Beside beside, hipStream_t st, SortedIds &out) {
  char *ws = (char *)workspace;
  const auto word = [&](uint64_t at) { return (uint32_t *)(ws + at); };
  SortPass p = {};
  p.n = plan.n, p.rows = plan.rows, p.bits = plan.bits, p.rounds = plan.rounds, p.counts = word(plan.counts_at), p.totals = word(plan.totals_at);
  p.blocks = plan.n <= kSmallSort ? (plan.n + kSmallOwn - 1) / kSmallOwn : plan.blocks;
  int to = 0;
  for (uint32_t pass = 0; pass < plan.passes; ++pass, to ^= 1) {
    p.keys = pass == 0 ? ids : word(plan.keys_at[to ^ 1]), p.at = pass == 0 ? nullptr : word(plan.at_at[to ^ 1]);
    p.out_keys = word(plan.keys_at[to]), p.out_at = word(plan.at_at[to]);
    p.shift = pass * plan.bits, p.hit = pass == 0 ? hit : nullptr;
    const uint32_t more = (plan.n <= kSmallSort || pass == 1) ? beside.blocks : 0;
    if (plan.n <= kSmallSort) {
      sort_small_kernel<<<p.blocks + more, kSmallThreads, 0, st>>>(p, beside);
    } else {
      sort_count_kernel<<<p.blocks + more, kSortThreads, 0, st>>>(p, beside);
      ANN_HIP(hipGetLastError());
      if (p.blocks <= kFewBlocks) {
        sort_place_kernel<false><<<p.blocks + more, kSortThreads, 0, st>>>(p, beside);
      } else {
        sort_scan_kernel<Beside><<<((1u << plan.bits) + 63) / 64, 1024, 0, st>>>(p);
        ANN_HIP(hipGetLastError());
        sort_place_kernel<true><<<p.blocks + more, kSortThreads, 0, st>>>(p, beside);
      }
    }
    ANN_HIP(hipGetLastError());
  }
  out.keys = word(plan.keys_at[to ^ 1]), out.positions = word(plan.at_at[to ^ 1]);
  return ANN_OK;
}

}  // namespace ann
