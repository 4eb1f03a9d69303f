// Sums of rows over runs of equal ids, in the order that id_sort gives: out[id] = sum of weight * row over the entries with that id, in fp32 in a fixed
// order; no atomic that a result depends on.
//
// Frequent ids make runs of any length, so runs do not go to lanes: lanes take a chunk of entries in order and sum them; the runs that lie
// within are written, the ends of runs that cross a border go to the workspace, from where a second kernel joins them in the borders' order.
// Bound by memory: every row is read once, several of them on their way at a time (80,000 x 768 bf16 into 17,000 fp32 rows: 45 us, 184 MB; the join 10 us of latency).
#pragma once
#include "id_sort.hpp"
#include "row_pieces.hpp"

namespace ann {

// Entries that are summed one after the other: few where there are few in all, so that the card has work (5,003 x 100: 28 us by 32 of them).
inline uint32_t chunk_entries(uint64_t n) { return n <= 16384 ? 8 : 32; }
constexpr uint32_t kMostChunks = 1 << 15;  // beyond, chunks are longer
constexpr uint32_t kFetched = 8;           // rows on their way at a time

struct Runs {
  const uint32_t *keys, *positions;  // in order; ids that are not below `ids` belong to nothing and come last
  uint32_t n, ids, chunk, chunks, dim;
  float *part;  // [chunks][2][part_ld]: the end of a run from the chunk before; the beginning of one that goes on in the next
  uint32_t part_ld;
};

struct RunsPlan {
  uint32_t chunk = 0, chunks = 0;
  uint64_t part_bytes = 0;
};
inline RunsPlan runs_plan(uint64_t n, uint32_t part_ld) {
  RunsPlan p;
  p.chunk = chunk_entries(n);
  while ((n + p.chunk - 1) / p.chunk > kMostChunks) p.chunk *= 2;
  p.chunks = (uint32_t)((n + p.chunk - 1) / p.chunk);
  p.part_bytes = ((uint64_t)p.chunks * 2 * part_ld * sizeof(float) + 255) / 256 * 256;
  return p;
}

// A group of LANES lanes takes a chunk and LANES * VEC columns; workgroups from `summing` on do the work beside.  Work:
//   kWeighted, kScalar        rows are weighted; a number to an entry is summed beside its row (column `dim` of the parts)
//   row(position)             an entry's row; weight(position), scalar(position)
//   write<VEC, END>(id, start, c, sum), write_scalar(id, start, sum)   a whole sum; start: the run's first entry, in order
//   beside(block, blocks)
template <typename T, int LANES, RowEnd END, typename Work>
__global__ __launch_bounds__(256) void runs_kernel(Runs g, Work work, uint32_t summing) {
  constexpr int VEC = 16 / (int)sizeof(T), kGroups = 256 / LANES;
  if (blockIdx.x >= summing) return work.beside(blockIdx.x - summing, gridDim.x - summing);
  const uint32_t tiles = g.dim ? (g.dim + LANES * VEC - 1) / (LANES * VEC) : 1, lane = threadIdx.x % LANES;
  const uint32_t at = blockIdx.x * kGroups + threadIdx.x / LANES, chunk = at / tiles;
  const uint32_t c = (at % tiles * LANES + lane) * VEC;
  if (chunk >= g.chunks) return;
  const uint32_t begin = chunk * g.chunk, end = begin + g.chunk < g.n ? begin + g.chunk : g.n;
  uint32_t id = g.keys[begin], start = begin;
  const uint32_t next = end < g.n ? g.keys[end] : 0xFFFFFFFFu;
  bool first = begin != 0 && g.keys[begin - 1] == id;  // the run began before this chunk
  float sum[VEC], scalar = 0.0f;
#pragma unroll
  for (int e = 0; e < VEC; ++e) sum[e] = 0.0f;
  const auto finish = [&](bool goes_on) {
    if (id >= g.ids) return;
    if (first || goes_on) {
      float *to = g.part + ((uint64_t)chunk * 2 + (first ? 0 : 1)) * g.part_ld;
#pragma unroll
      for (int e = 0; e < VEC; ++e)
        if (END == kWholePieces ? c < g.dim : c + e < g.dim) to[c + e] = sum[e];
      if (Work::kScalar && c == 0) to[g.dim] = scalar;
    } else {
      if (c < g.dim) work.template write<VEC, END>(id, start, c, sum);
      if (Work::kScalar && c == 0) work.write_scalar(id, start, scalar);
    }
  };
  for (uint32_t i0 = begin; i0 < end; i0 += LANES) {
    // an entry to a lane, handed round
    const uint32_t mine = i0 + lane < end ? i0 + lane : end - 1;
    const uint32_t my_key = g.keys[mine], my_position = g.positions[mine];
    const uint64_t my_row = (uint64_t)work.row(my_position);
    const float my_weight = Work::kWeighted ? work.weight(my_position) : 1.0f, my_scalar = Work::kScalar ? work.scalar(my_position) : 0.0f;
    const auto of = [&](uint32_t u, uint32_t v) {
      if constexpr (LANES == kWave)
        return (uint32_t)__builtin_amdgcn_readlane((int)v, (int)u);
      else
        return (uint32_t)__builtin_amdgcn_ds_bpermute(((int)(lane_id() / LANES * LANES) + (int)u) << 2, (int)v);
    };
    const uint32_t here = end - i0 < LANES ? end - i0 : LANES;
    for (uint32_t u0 = 0; u0 < here; u0 += kFetched) {
      RowPiece<T, VEC, END> v[kFetched];
      uint32_t key[kFetched];
      float weight[kFetched], number[kFetched];
#pragma unroll
      for (uint32_t u = 0; u < kFetched; ++u) {
        // (behind the last entry: the last one's once more)
        key[u] = of(u0 + u, my_key);
        if (Work::kWeighted) weight[u] = __uint_as_float(of(u0 + u, __float_as_uint(my_weight)));
        if (Work::kScalar) number[u] = __uint_as_float(of(u0 + u, __float_as_uint(my_scalar)));
        const uint64_t row = of(u0 + u, (uint32_t)my_row) | (uint64_t)of(u0 + u, (uint32_t)(my_row >> 32)) << 32;
        v[u].load((const T *)row, c, g.dim);
      }
#pragma unroll
      for (uint32_t u = 0; u < kFetched; ++u) {
        if (u0 + u >= here || key[u] >= g.ids) continue;  // (what belongs to nothing comes last)
        if (key[u] != id) {
          finish(false);
          id = key[u], start = i0 + u0 + u, first = false, scalar = 0.0f;
#pragma unroll
          for (int e = 0; e < VEC; ++e) sum[e] = 0.0f;
        }
        if (Work::kScalar) scalar += number[u];
#pragma unroll
        for (int e = 0; e < VEC; ++e) sum[e] = Work::kWeighted ? __builtin_fmaf(weight[u], v[u].get(e), sum[e]) : sum[e] + v[u].get(e);
      }
    }
  }
  finish(id == next);
}

// Runs that cross borders between chunks, by the chunk in which they begin, 256 columns at a time: a wavefront to a border, which joins the runs of
// few chunks alone; those of many are shared out over the workgroup's wavefronts afterwards, one after the other.  (A workgroup to a border:
// 12 us for 2,500 borders of which one in two begins nothing or a run of two chunks; with four wavefronts 23 us where one id in ten is alike.)
constexpr uint32_t kJoinWaves = 8, kJoinAlone = 8;
template <typename Work>
__global__ __launch_bounds__(kJoinWaves * 64) void runs_join_kernel(Runs g, Work work) {
  __shared__ float room[kJoinWaves - 1][256];
  __shared__ uint32_t starts[kJoinWaves], counts[kJoinWaves];
  const uint32_t lane = threadIdx.x % 64, wave = threadIdx.x / 64, c = blockIdx.y * 256 + lane, columns = g.dim + (Work::kScalar ? 1 : 0);
  // sums of parts from .. to - 1 of the chunks behind `chunk`, and its own
  const auto add_parts = [&](float (&sum)[4], uint32_t from, uint32_t to) {
    for (uint32_t k = from; k < to; k += 8) {
      float v[8][4];
#pragma unroll
      for (uint32_t u = 0; u < 8; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e) v[u][e] = k + u < to && c + e * 64 < columns ? g.part[(uint64_t)(k + u) * 2 * g.part_ld + c + e * 64] : 0.0f;
#pragma unroll
      for (uint32_t u = 0; u < 8; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e] += v[u][e];
    }
  };
  const auto begin_with = [&](float (&sum)[4], uint32_t chunk, bool own) {
#pragma unroll
    for (int e = 0; e < 4; ++e) sum[e] = own && c + e * 64 < columns ? g.part[((uint64_t)chunk * 2 + 1) * g.part_ld + c + e * 64] : 0.0f;
  };
  const auto write = [&](uint32_t id, uint32_t start, int e, float v) {
    const float total[1] = {v};
    if (c + e * 64 >= columns) return;
    if (Work::kScalar && c + e * 64 == g.dim)
      work.write_scalar(id, start, v);
    else
      work.template write<1, kByElement>(id, start, c + e * 64, total);
  };
  const uint32_t mine = blockIdx.x * kJoinWaves + wave;  // the border behind this chunk
  uint32_t start = 0, count = 0;                         // of a run that begins in it and goes on: its first entry, and the chunks that it goes on in
  if (mine + 1 < g.chunks) {
    const uint32_t border = (mine + 1) * g.chunk, begin = mine * g.chunk;
    const uint32_t before = begin ? g.keys[begin - 1] : 0xFFFFFFFFu, ends = g.keys[border - 1], id = g.keys[border];  // (read side by side)
    if (id < g.ids && ends == id && before != id) {
      count = 1;
      for (;;) {
        const uint64_t next = (uint64_t)mine + 1 + count + lane;
        const uint64_t with = __ballot(next < g.chunks && g.keys[next * g.chunk] == id);
        if (with != ~0ull) {
          count += __builtin_ctzll(~with);
          break;
        }
        count += 64;
      }
      for (uint32_t i0 = begin;; i0 += 64) {
        const uint64_t with = __ballot(i0 + lane < border && g.keys[i0 + lane] == id);
        if (with) {
          start = i0 + __builtin_ctzll(with);
          break;
        }
      }
      if (count <= kJoinAlone) {
        float sum[4];
        begin_with(sum, mine, true);
        add_parts(sum, mine + 1, mine + 1 + count);
#pragma unroll
        for (int e = 0; e < 4; ++e) write(id, start, e, sum[e]);
        count = 0;
      }
    }
  }
  if (lane == 0) starts[wave] = start, counts[wave] = count;
  __syncthreads();
  for (uint32_t w = 0; w < kJoinWaves; ++w) {
    const uint32_t chunk = blockIdx.x * kJoinWaves + w, of = counts[w];
    if (of == 0) continue;
    float sum[4];
    begin_with(sum, chunk, wave == 0);
    add_parts(sum, chunk + 1 + (uint32_t)((uint64_t)of * wave / kJoinWaves), chunk + 1 + (uint32_t)((uint64_t)of * (wave + 1) / kJoinWaves));
    if (wave != 0) {
#pragma unroll
      for (int e = 0; e < 4; ++e) room[wave - 1][lane + e * 64] = sum[e];
    }
    __syncthreads();
    if (wave == 0) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
#pragma unroll
        for (uint32_t o = 0; o < kJoinWaves - 1; ++o) sum[e] += room[o][lane + e * 64];
        write(g.keys[(uint64_t)(chunk + 1) * g.chunk], starts[w], e, sum[e]);
      }
    }
    __syncthreads();
  }
}

// Both kernels; `beside` workgroups more in the first.
template <typename T, typename Work>
static ann_status sum_runs(const Runs &g, const Work &work, uint32_t beside, hipStream_t st) {
  constexpr uint32_t VEC = 16 / sizeof(T);
  const auto sums = [&](auto lanes, auto end) {
    constexpr uint32_t L = decltype(lanes)::value;
    const uint64_t groups = (uint64_t)g.chunks * (g.dim ? (g.dim + L * VEC - 1) / (L * VEC) : 1);
    const uint32_t summing = (uint32_t)((groups * L + 255) / 256);
    runs_kernel<T, L, decltype(end)::value><<<summing + beside, 256, 0, st>>>(g, work, summing);
  };
  const auto sums_of = [&](auto lanes) {
    if (g.dim % VEC == 0)
      sums(lanes, std::integral_constant<RowEnd, kWholePieces>());
    else
      sums(lanes, std::integral_constant<RowEnd, kShifted>());
  };
  if (g.dim <= 16 * VEC)
    sums_of(std::integral_constant<int, 16>());
  else
    sums_of(std::integral_constant<int, 64>());
  ANN_HIP(hipGetLastError());
  if (g.chunks > 1) {
    runs_join_kernel<<<dim3((g.chunks - 1 + kJoinWaves - 1) / kJoinWaves, (g.dim + (Work::kScalar ? 1 : 0) + 255) / 256), kJoinWaves * 64, 0, st>>>(g, work);
    ANN_HIP(hipGetLastError());
  }
  return ANN_OK;
}

}  // namespace ann
