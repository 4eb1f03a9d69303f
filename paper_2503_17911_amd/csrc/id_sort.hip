// A stable radix sort of ids with their positions, from the lowest digit up: two or three passes of up to 11 bits.
//
// A pass counts the digits of every block's entries, then every block places its entries behind the smaller digits' and the earlier blocks'.
// The place within a block follows the entries' order (a wavefront finds the lanes with its digit by one ballot to a bit, and counts
// rounds and wavefronts one after the other), so equal ids stay in the order of their positions and the result does not depend on
// timing.  With few blocks a block adds up the counts of the others itself; with many a kernel between the two does.  Up to kSmallSort entries
// are sorted by one workgroup in LDS.  Bound by launches and the counters' latency: 80,000 ids are 320 KB.
#include "id_sort.hpp"

#include "device_utils.hpp"

namespace ann {

constexpr uint32_t kSortThreads = 256, kSortWaves = kSortThreads / kWave, kSortRounds = 8;
constexpr uint32_t kMaxBits = 11, kMaxDigits = 1u << kMaxBits;
constexpr uint32_t kFewBlocks = 64;      // up to so many, a block adds the others' counts itself
constexpr uint32_t kMostBlocks = 4096;   // beyond, blocks take more rounds
constexpr uint32_t kSmallThreads = 1024;

IdSortPlan id_sort_plan(uint64_t n, uint64_t rows) {
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
  uint32_t *out_keys, *out_at, *counts, *totals, *hit;
  uint32_t n, rows, shift, bits, rounds;
};

__device__ __forceinline__ uint32_t sort_key(const SortPass &p, uint32_t i) {
  const uint32_t key = p.keys[i];
  return !p.at && key > p.rows ? p.rows : key;
}

// counts[block][digit]
__global__ __launch_bounds__(kSortThreads) void sort_count_kernel(SortPass p) {
  __shared__ uint32_t count[kMaxDigits];
  const uint32_t digits = 1u << p.bits, first = blockIdx.x * p.rounds * kSortThreads;
  for (uint32_t d = threadIdx.x; d < digits; d += kSortThreads) count[d] = 0;
  if (p.hit)
    for (uint64_t w = (uint64_t)blockIdx.x * kSortThreads + threadIdx.x; w < (p.rows + 31ull) / 32; w += (uint64_t)gridDim.x * kSortThreads) p.hit[w] = 0;
  __syncthreads();
  for (uint32_t r = 0; r < p.rounds; ++r) {
    const uint64_t i = (uint64_t)first + r * kSortThreads + threadIdx.x;
    if (i < p.n) atomicAdd(&count[sort_key(p, (uint32_t)i) >> p.shift & (digits - 1)], 1u);
  }
  __syncthreads();
  for (uint32_t d = threadIdx.x; d < digits; d += kSortThreads) p.counts[(uint64_t)blockIdx.x * digits + d] = count[d];
}

// counts[block][digit] becomes the sum over the blocks before; totals[digit] that over all.  64 digits to a workgroup, 16 runs of blocks.
__global__ __launch_bounds__(1024) void sort_scan_kernel(SortPass p, uint32_t blocks) {
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
template <bool SCANNED>
__global__ __launch_bounds__(kSortThreads) void sort_place_kernel(SortPass p) {
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
#pragma unroll 8
        for (uint32_t b = 0; b < gridDim.x; ++b) {
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
  for (uint32_t r = 0; r < p.rounds; ++r) {
    const uint64_t i = first + r * kWave + lane;
    if (i < p.n) atomicAdd(&of_wave[wave][sort_key(p, (uint32_t)i) >> p.shift & (digits - 1)], 1u);
  }
  __syncthreads();
  for (uint32_t d = threadIdx.x; d < digits; d += kSortThreads) {
    uint32_t at = place[d];
    for (uint32_t w = 0; w < kSortWaves; ++w) {
      const uint32_t c = of_wave[w][d];
      of_wave[w][d] = at;
      at += c;
    }
  }
  __syncthreads();
  for (uint32_t r = 0; r < p.rounds; ++r) {
    const uint64_t i = first + r * kWave + lane;
    const bool there = i < p.n;
    const uint32_t key = there ? sort_key(p, (uint32_t)i) : 0, at = there ? (p.at ? p.at[i] : (uint32_t)i) : 0;
    const uint32_t digit = key >> p.shift & (digits - 1);
    const uint64_t same = lanes_with(digit, there, digit, p.bits);
    const uint32_t rank = __popcll(same & ((1ull << lane) - 1));
    if (there) {
      const uint32_t to = of_wave[wave][digit] + rank;
      p.out_keys[to] = key, p.out_at[to] = at;
      if (p.hit && key < p.rows && rank == 0) atomicOr(&p.hit[key / 32], 1u << (key % 32));
    }
    // the first of the lanes with the digit moves its place on, once all have read it
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    if (there && rank == 0) of_wave[wave][digit] += __popcll(same);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
}

// Up to kSmallSort entries: passes of 4 bits within one workgroup, four entries to a lane, in LDS.
__global__ __launch_bounds__(kSmallThreads) void sort_small_kernel(SortPass p) {
  constexpr uint32_t kDigits = 16, kWaves = kSmallThreads / kWave, kEach = kSmallSort / kSmallThreads;
  __shared__ uint32_t keys[2][kSmallSort], at[2][kSmallSort], count[kDigits * kWaves + 1], room[kWaves + 1];
  const uint32_t wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
  for (uint32_t i = threadIdx.x; i < kSmallSort; i += kSmallThreads) {
    keys[0][i] = i < p.n ? sort_key(p, i) : 0xFFFFFFFFu;  // (behind all others, where they stay)
    at[0][i] = i;
  }
  __syncthreads();
  uint32_t from = 0;
  for (uint32_t shift = 0; shift < p.bits; shift += 4, from ^= 1) {
    // a wavefront takes kEach * 64 entries side by side, 64 at a time
    uint32_t key[kEach], place[kEach], digit[kEach], mine = 0;  // mine: lane d < 16 counts the wavefront's entries of digit d
#pragma unroll
    for (uint32_t r = 0; r < kEach; ++r) {
      const uint32_t i = (wave * kEach + r) * kWave + lane;
      key[r] = keys[from][i], place[r] = at[from][i];
      digit[r] = key[r] >> shift & (kDigits - 1);
    }
    uint64_t same[kEach];
    uint32_t before[kEach];  // entries of its digit in the wavefront's earlier rounds
#pragma unroll
    for (uint32_t r = 0; r < kEach; ++r) {
      same[r] = lanes_with(digit[r], true, digit[r], 4);
      before[r] = (uint32_t)__builtin_amdgcn_ds_bpermute((int)digit[r] << 2, (int)mine);
      mine += __popcll(lanes_with(digit[r], true, lane % kDigits, 4));
    }
    if (lane < kDigits) count[lane * kWaves + wave] = mine;
    __syncthreads();
    // places: by digit, then by wavefront
    uint32_t all;
    const uint32_t v = threadIdx.x < kDigits * kWaves ? count[threadIdx.x] : 0;
    const uint32_t start = exclusive_sum<kSmallThreads>(v, room, all);
    if (threadIdx.x < kDigits * kWaves) count[threadIdx.x] = start;
    __syncthreads();
#pragma unroll
    for (uint32_t r = 0; r < kEach; ++r) {
      const uint32_t to = count[digit[r] * kWaves + wave] + before[r] + __popcll(same[r] & ((1ull << lane) - 1));
      keys[from ^ 1][to] = key[r], at[from ^ 1][to] = place[r];
    }
    __syncthreads();
  }
  for (uint32_t i = threadIdx.x; i < p.n; i += kSmallThreads) {
    p.out_keys[i] = keys[from][i], p.out_at[i] = at[from][i];
  }
}

ann_status sort_ids(const IdSortPlan &plan, const uint32_t *ids, void *workspace, uint32_t *hit, hipStream_t st, SortedIds &out) {
  char *ws = (char *)workspace;
  const auto word = [&](uint64_t at) { return (uint32_t *)(ws + at); };
  SortPass p = {};
  p.n = plan.n, p.rows = plan.rows, p.bits = plan.bits, p.rounds = plan.rounds, p.counts = word(plan.counts_at), p.totals = word(plan.totals_at);
  int to = 0;
  for (uint32_t pass = 0; pass < plan.passes; ++pass, to ^= 1) {
    p.keys = pass == 0 ? ids : word(plan.keys_at[to ^ 1]), p.at = pass == 0 ? nullptr : word(plan.at_at[to ^ 1]);
    p.out_keys = word(plan.keys_at[to]), p.out_at = word(plan.at_at[to]);
    p.shift = pass * plan.bits, p.hit = pass == 0 ? hit : nullptr;
    if (plan.n <= kSmallSort) {
      sort_small_kernel<<<1, kSmallThreads, 0, st>>>(p);
    } else {
      sort_count_kernel<<<plan.blocks, kSortThreads, 0, st>>>(p);
      ANN_HIP(hipGetLastError());
      if (plan.blocks <= kFewBlocks) {
        sort_place_kernel<false><<<plan.blocks, kSortThreads, 0, st>>>(p);
      } else {
        sort_scan_kernel<<<((1u << plan.bits) + 63) / 64, 1024, 0, st>>>(p, plan.blocks);
        ANN_HIP(hipGetLastError());
        sort_place_kernel<true><<<plan.blocks, kSortThreads, 0, st>>>(p);
      }
    }
    ANN_HIP(hipGetLastError());
  }
  out.keys = word(plan.keys_at[to ^ 1]), out.positions = word(plan.at_at[to ^ 1]);
  return ANN_OK;
}

}  // namespace ann
