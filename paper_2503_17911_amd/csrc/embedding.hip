// Rows of a table by their ids, times a scale, and the table's gradient.
//
//   y[i] = scale * table[ids[i]];   dtable[r] = scale * sum over i with ids[i] = r of dy[i]
//
// Bound by memory.  Forward: a row belongs to 16 or 64 lanes, pieces of 16 bytes of the output with any alignment.  Gradient: the ids
// are put in order with their positions (id_sort), so that a table's row is a run of entries and its sum has a fixed order; no
// atomic that a result depends on.  Frequent ids make runs of any length, so runs do not go to lanes: lanes take a chunk of entries in
// order, sums them in fp32 and writes the runs that lie within; the ends of runs that cross a border go to the workspace, from where a
// second kernel joins them in the borders' order.  Rows without an id are filled with zeros beside the sums (a bit to a row
// says which; few ids: the whole table is filled beside the sorting).
#include "id_sort.hpp"
#include "row_pieces.hpp"

namespace ann {

// Entries that are summed one after the other: few where there are few in all, so that the card has work (5,003 x 100: 28 us by 32 of them).
static uint32_t chunk_entries(uint64_t n) { return n <= 8192 ? 8 : n <= 16384 ? 16 : 32; }
constexpr uint32_t kMostChunks = 1 << 15;  // beyond, chunks are longer
constexpr uint32_t kFetched = 8;         // rows on their way at a time

struct EmbedArgs {
  const void *from;  // forward: the table; backward: dy
  void *to;          // forward: y; backward: dtable
  const uint32_t *ids;
  uint64_t n, rows, from_stride, to_stride;
  uint32_t dim;
  float scale;
  // backward
  const uint32_t *keys, *positions;
  const uint8_t *hit;
  float *part;  // [chunks][2][dim]: the end of a run from the chunk before; the beginning of one that goes on in the next
  uint32_t chunk, chunks, accumulate;
};

// F: the table's type, T: of y.  A group of LANES lanes takes kUnits pieces to a lane at a time, `slots` of them to a row: so many reads are on
// their way at once (one after the other: 72 us for 80,000 x 960 fp32 to bf16).
template <typename F, typename T, int LANES, RowEnd END>
__global__ __launch_bounds__(256) void embed_kernel(EmbedArgs g, uint32_t slots) {
  constexpr int VEC = 16 / (int)sizeof(T), kGroups = 256 / LANES, kParts = VEC * (int)sizeof(F) / 16, kEach = VEC / kParts, kUnits = 4;
  const uint32_t lane = threadIdx.x % LANES;
  const uint64_t units = g.n * slots;
  for (uint64_t u0 = ((uint64_t)blockIdx.x * kGroups + threadIdx.x / LANES) * kUnits; u0 < units; u0 += (uint64_t)gridDim.x * kGroups * kUnits) {
    uint64_t row[kUnits];
    uint32_t c[kUnits], id[kUnits];
    row[0] = u0 / slots;
    uint32_t slot = (uint32_t)(u0 % slots);
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      if (u) {
        const bool next = ++slot == slots;
        row[u] = row[u - 1] + next;
        slot = next ? 0 : slot;
      }
      c[u] = row[u] < g.n ? (slot * LANES + lane) * VEC : g.dim;
      id[u] = g.ids[row[u] < g.n ? row[u] : g.n - 1];
    }
    RowPiece<F, kEach, END> v[kUnits][kParts];
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      const F *from = (const F *)g.from + (id[u] < g.rows ? id[u] : 0) * g.from_stride;  // (there is a row)
#pragma unroll
      for (int p = 0; p < kParts; ++p) v[u][p].load(from, c[u] + p * kEach, g.dim);
    }
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      float f[VEC];
#pragma unroll
      for (int e = 0; e < VEC; ++e) f[e] = id[u] < g.rows ? v[u][e / kEach].get(e % kEach) * g.scale : 0.0f;
      RowPiece<T, VEC, END> o;
      o.set(f);
      o.store((T *)g.to + row[u] * g.to_stride, c[u], g.dim);
    }
  }
}

// Rows of zeros; hit: but those whose bit is set.
template <typename F>
__device__ __forceinline__ void zero_rows(F *table, uint64_t first, uint64_t end, uint64_t stride, uint32_t dim, const uint8_t *hit, uint32_t block,
                                          uint32_t blocks) {
  constexpr int VEC = 16 / (int)sizeof(F);
  const uint32_t waves = blockDim.x / kWave;
  RowPiece<F, VEC> zero;
  zero.clear();
  for (uint64_t r = first + (uint64_t)block * waves + threadIdx.x / kWave; r < end; r += (uint64_t)blocks * waves) {
    if (hit && hit[r]) continue;
    for (uint32_t c = threadIdx.x % kWave * VEC; c < dim; c += kWave * VEC) zero.store(table + r * stride, c, dim);
  }
}
template <typename F>
__global__ __launch_bounds__(256) void embed_zero_kernel(F *table, uint64_t rows, uint64_t stride, uint32_t dim) {
  zero_rows<F>(table, 0, rows, stride, dim, nullptr, blockIdx.x, gridDim.x);
}

// Zeros beside the sorting: few ids, all rows, before any other is written; many, the rows that no id names, `early` of them beside the second
// pass' counting, which is the shorter of its kernels.
template <typename F>
struct ZeroBeside {
  uint32_t blocks, dim;
  F *table;
  uint64_t rows, early, stride;
  const uint8_t *hit;
  __device__ __forceinline__ void operator()(uint32_t stage, uint32_t part, uint32_t parts) const {
    zero_rows<F>(table, stage == 2 ? early : 0, stage == 1 ? early : rows, stride, dim, stage ? hit : nullptr, part, parts);
  }
};

template <typename F, int VEC, RowEnd END>
__device__ __forceinline__ void write_gradient(const EmbedArgs &g, uint32_t row, uint32_t c, const float (&sum)[VEC]) {
  F *to = (F *)g.to + row * g.to_stride;
  if constexpr (VEC == 1) {
    to[c] = from_f32<F>(g.accumulate ? __builtin_fmaf(sum[0], g.scale, to_f32(to[c])) : sum[0] * g.scale);
  } else {
    constexpr int kEach = 16 / (int)sizeof(F), N = VEC < kEach ? VEC : kEach;
#pragma unroll
    for (int p = 0; p < VEC; p += N) {
      RowPiece<F, N, END> o;
      float v[N];
      if (g.accumulate) o.load(to, c + p, g.dim);
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] = g.accumulate ? __builtin_fmaf(sum[p + e], g.scale, o.get(e)) : sum[p + e] * g.scale;
      o.set(v);
      o.store(to, c + p, g.dim);
    }
  }
}

// T: of dy, F: of the table.  A group of LANES lanes takes a chunk and LANES * VEC columns.  Workgroups from `summing` on write zeros.
template <typename T, typename F, int LANES, RowEnd END>
__global__ __launch_bounds__(256) void embed_grad_kernel(EmbedArgs g, uint32_t summing) {
  constexpr int VEC = 16 / (int)sizeof(T), kGroups = 256 / LANES;
  if (blockIdx.x >= summing) {
    zero_rows<F>((F *)g.to, 0, g.rows, g.to_stride, g.dim, g.hit, blockIdx.x - summing, gridDim.x - summing);
    return;
  }
  const uint32_t tiles = (g.dim + LANES * VEC - 1) / (LANES * VEC), lane = threadIdx.x % LANES;
  const uint32_t at = blockIdx.x * kGroups + threadIdx.x / LANES, chunk = at / tiles;
  const uint32_t c = (at % tiles * LANES + lane) * VEC;
  if (chunk >= g.chunks) return;
  const uint32_t begin = chunk * g.chunk, end = begin + g.chunk < g.n ? begin + g.chunk : (uint32_t)g.n;
  uint32_t row = g.keys[begin];
  const uint32_t next = end < g.n ? g.keys[end] : 0xFFFFFFFFu;
  bool first = begin != 0 && g.keys[begin - 1] == row;  // the run began before this chunk
  float sum[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) sum[e] = 0.0f;
  const auto finish = [&](bool goes_on) {
    if (row >= g.rows || c >= g.dim) return;
    if (first || goes_on) {
      float *to = g.part + ((uint64_t)chunk * 2 + (first ? 0 : 1)) * g.dim + c;
#pragma unroll
      for (int e = 0; e < VEC; ++e)
        if (END == kWholePieces || c + e < g.dim) to[e] = sum[e];
    } else {
      write_gradient<F, VEC, END>(g, row, c, sum);
    }
  };
  for (uint32_t i0 = begin; i0 < end; i0 += LANES) {
    // an entry to a lane, handed round
    const uint32_t mine = i0 + lane < end ? i0 + lane : end - 1;
    const uint32_t my_key = g.keys[mine], my_position = g.positions[mine];
    const uint32_t here = end - i0 < LANES ? end - i0 : LANES;
    for (uint32_t u0 = 0; u0 < here; u0 += kFetched) {
      RowPiece<T, VEC, END> v[kFetched];
      uint32_t key[kFetched];
#pragma unroll
      for (uint32_t u = 0; u < kFetched; ++u) {
        // (behind the last entry: the last one's once more)
        uint32_t position;
        if constexpr (LANES == kWave) {
          key[u] = (uint32_t)__builtin_amdgcn_readlane((int)my_key, (int)(u0 + u)), position = (uint32_t)__builtin_amdgcn_readlane((int)my_position, (int)(u0 + u));
        } else {
          const int from = ((int)(lane_id() / LANES * LANES) + (int)(u0 + u)) << 2;
          key[u] = (uint32_t)__builtin_amdgcn_ds_bpermute(from, (int)my_key), position = (uint32_t)__builtin_amdgcn_ds_bpermute(from, (int)my_position);
        }
        v[u].load((const T *)g.from + position * g.from_stride, c, g.dim);
      }
#pragma unroll
      for (uint32_t u = 0; u < kFetched; ++u) {
        if (u0 + u >= here || key[u] >= g.rows) continue;  // (what belongs to no row comes last)
        if (key[u] != row) {
          finish(false);
          row = key[u], first = false;
#pragma unroll
          for (int e = 0; e < VEC; ++e) sum[e] = 0.0f;
        }
#pragma unroll
        for (int e = 0; e < VEC; ++e) sum[e] += v[u].get(e);
      }
    }
  }
  finish(row == next);
}

// Runs that cross borders between chunks, by the chunk in which they begin: 256 columns to a workgroup of four wavefronts, which share out
// the run's chunks.
template <typename F>
__global__ __launch_bounds__(256) void embed_join_kernel(EmbedArgs g) {
  __shared__ float room[3][256];
  const uint32_t chunk = blockIdx.x, border = (chunk + 1) * g.chunk, begin = chunk * g.chunk;
  // (read side by side: most workgroups end here)
  const uint32_t before = begin ? g.keys[begin - 1] : 0xFFFFFFFFu, last_key = g.keys[border - 1], row = g.keys[border];
  if (row >= g.rows || last_key != row || before == row) return;
  const uint32_t lane = threadIdx.x % 64, wave = threadIdx.x / 64, c = blockIdx.y * 256 + lane;
  uint32_t last = chunk + 1;  // the last chunk that begins with the run
  for (;;) {
    const uint32_t next = last + 1 + lane;
    const uint64_t with = __ballot(next < g.chunks && g.keys[next * g.chunk] == row);
    if (with != ~0ull) {
      last += __builtin_ctzll(~with);
      break;
    }
    last += 64;
  }
  const uint32_t count = last - chunk, from = chunk + 1 + (uint32_t)((uint64_t)count * wave / 4), to = chunk + 1 + (uint32_t)((uint64_t)count * (wave + 1) / 4);
  float sum[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) sum[e] = wave == 0 && c + e * 64 < g.dim ? g.part[((uint64_t)chunk * 2 + 1) * g.dim + c + e * 64] : 0.0f;
  for (uint32_t k = from; k < to; k += 8) {
    float v[8][4];
#pragma unroll
    for (uint32_t u = 0; u < 8; ++u)
#pragma unroll
      for (int e = 0; e < 4; ++e) v[u][e] = k + u < to && c + e * 64 < g.dim ? g.part[(uint64_t)(k + u) * 2 * g.dim + c + e * 64] : 0.0f;
#pragma unroll
    for (uint32_t u = 0; u < 8; ++u)
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[e] += v[u][e];
  }
  if (wave != 0) {
#pragma unroll
    for (int e = 0; e < 4; ++e) room[wave - 1][lane + e * 64] = sum[e];
  }
  __syncthreads();
  if (wave != 0) return;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if (c + e * 64 >= g.dim) break;
    const float total[1] = {((sum[e] + room[0][lane + e * 64]) + room[1][lane + e * 64]) + room[2][lane + e * 64]};
    write_gradient<F, 1, kByElement>(g, row, c + e * 64, total);
  }
}

struct EmbedGradPlan {
  IdSortPlan sort;
  uint32_t chunk = 0, chunks = 0;
  uint64_t part_at = 0, hit_at = 0, bytes = 0;
};

static EmbedGradPlan embed_grad_plan(uint64_t n, uint64_t rows, uint32_t dim) {
  EmbedGradPlan p;
  if (n == 0) return p;
  p.sort = id_sort_plan(n, rows);
  p.chunk = chunk_entries(n);
  while ((n + p.chunk - 1) / p.chunk > kMostChunks) p.chunk *= 2;
  p.chunks = (uint32_t)((n + p.chunk - 1) / p.chunk);
  p.part_at = p.sort.bytes;
  p.hit_at = p.part_at + ((uint64_t)p.chunks * 2 * dim * sizeof(float) + 255) / 256 * 256;
  p.bytes = p.hit_at + (n > kSmallSort ? (rows + 255) / 256 * 256 : 0);
  return p;
}

static ann_status check_embedding(const char *what, uint64_t n, uint64_t rows, uint32_t dim, uint32_t table_type, uint32_t type) {
  if (type > ANN_BF16) return fail(ANN_EINVAL, "%s: unknown type %u", what, type);
  if (table_type != type && table_type != ANN_F32) return fail(ANN_EINVAL, "%s: tables are of the rows' type or ANN_F32, not %u", what, table_type);
  if (dim == 0) return fail(ANN_EINVAL, "%s: dim == 0", what);
  if (dim > ANN_MAX_NORM_DIM) return fail(ANN_ECAPACITY, "%s: dim = %u exceeds ANN_MAX_NORM_DIM = %u", what, dim, ANN_MAX_NORM_DIM);
  if (n >= (1ull << 31) || rows > (1ull << 31)) return fail(ANN_ECAPACITY, "%s: n below 2^31 and at most 2^31 rows", what);
  return ANN_OK;
}

template <typename T, typename F>
static ann_status embedding_backward(const EmbedGradPlan &p, EmbedArgs g, char *ws, hipStream_t st) {
  uint8_t *hit = (uint8_t *)(ws + p.hit_at);
  if (g.n == 0 || g.rows == 0) {
    if (g.rows == 0 || g.accumulate) return ANN_OK;
    embed_zero_kernel<F><<<(uint32_t)(g.rows < 8192 ? (g.rows + 3) / 4 : 2048), 256, 0, st>>>((F *)g.to, g.rows, g.to_stride, g.dim);
    ANN_HIP(hipGetLastError());
    return ANN_OK;
  }
  const bool small = g.n <= kSmallSort, beside = !g.accumulate && (small || p.sort.passes > 1), fill = !g.accumulate && !beside;
  // (two workgroups of 512 lanes to a compute unit, beside the sort's few; with few ids as many of 1,024 lanes as have a row each lane group)
  const uint64_t most = small ? 256 : 768, by_rows = (g.rows + (small ? 15 : 7)) / (small ? 16 : 8);
  const uint32_t zero_blocks = (uint32_t)(by_rows < most ? by_rows : most);
  const ZeroBeside<F> zeros = {beside ? zero_blocks : 0, g.dim, (F *)g.to, g.rows, g.rows * 2 / 5, g.to_stride, hit};
  SortedIds sorted;
  if (ann_status s = sort_ids(p.sort, g.ids, ws, small || g.accumulate ? nullptr : hit, zeros, st, sorted)) return s;
  g.keys = sorted.keys, g.positions = sorted.positions, g.hit = hit, g.part = (float *)(ws + p.part_at), g.chunk = p.chunk, g.chunks = p.chunks;
  constexpr uint32_t VEC = 16 / sizeof(T);
  const auto sums = [&](auto lanes, auto end) {
    constexpr uint32_t L = decltype(lanes)::value;
    const uint64_t groups = (uint64_t)p.chunks * ((g.dim + L * VEC - 1) / (L * VEC));
    const uint32_t summing = (uint32_t)((groups * L + 255) / 256);
    embed_grad_kernel<T, F, L, decltype(end)::value><<<summing + (fill ? zero_blocks : 0), 256, 0, st>>>(g, summing);
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
  if (p.chunks > 1) {
    embed_join_kernel<F><<<dim3(p.chunks - 1, (g.dim + 255) / 256), 256, 0, st>>>(g);
    ANN_HIP(hipGetLastError());
  }
  return ANN_OK;
}

}  // namespace ann

using namespace ann;

extern "C" ann_status ann_embedding(const void *table, uint64_t rows, uint32_t dim, uint64_t table_stride, uint32_t table_type, const uint32_t *ids,
                                    uint64_t n, float scale, void *y, uint64_t y_stride, uint32_t type, void *stream) {
  if (ann_status s = check_embedding("ann_embedding", n, rows, dim, table_type, type)) return s;
  if (n == 0) return ANN_OK;
  if ((rows && !table) || !ids || !y) return fail(ANN_EINVAL, "ann_embedding: NULL argument");
  if ((rows && table_stride < dim) || y_stride < dim) return fail(ANN_EINVAL, "ann_embedding: a row stride is shorter than a row");
  EmbedArgs g = {};
  g.from = table, g.to = y, g.ids = ids, g.n = n, g.rows = rows, g.from_stride = table_stride, g.to_stride = y_stride, g.dim = dim, g.scale = scale;
  const hipStream_t st = (hipStream_t)stream;
  const auto run = [&](auto f, auto t) {
    typedef decltype(f) F;
    typedef decltype(t) T;
    if (rows == 0) {  // (padding alone)
      embed_zero_kernel<T><<<(uint32_t)(n < 8192 ? (n + 3) / 4 : 2048), 256, 0, st>>>((T *)y, n, y_stride, dim);
      return;
    }
    constexpr uint32_t VEC = 16 / sizeof(T);
    const auto as = [&](auto lanes, auto end) {
      constexpr uint32_t L = decltype(lanes)::value;
      const uint32_t slots = (dim + L * VEC - 1) / (L * VEC);
      const uint64_t groups = (n * slots + 3) / 4, want = (groups * L + 255) / 256;
      embed_kernel<F, T, L, decltype(end)::value><<<(uint32_t)(want < 65536 ? want : 65536), 256, 0, st>>>(g, slots);
    };
    const auto with_lanes = [&](auto lanes) {
      if (dim % VEC == 0)
        as(lanes, std::integral_constant<RowEnd, kWholePieces>());
      else
        as(lanes, std::integral_constant<RowEnd, kShifted>());
    };
    if (dim <= 16 * VEC)
      with_lanes(std::integral_constant<int, 16>());
    else if (dim % (64 * VEC) > 32 * VEC || dim % (64 * VEC) == 0 || dim > 512 * VEC)
      with_lanes(std::integral_constant<int, 64>());
    else
      with_lanes(std::integral_constant<int, 32>());
  };
  if (type == ANN_F32)
    run(0.0f, 0.0f);
  else if (type == ANN_F16)
    table_type == ANN_F32 ? run(0.0f, f16_t()) : run(f16_t(), f16_t());
  else
    table_type == ANN_F32 ? run(0.0f, bf16_t()) : run(bf16_t(), bf16_t());
  ANN_HIP(hipGetLastError());
  return ANN_OK;
}

extern "C" uint64_t ann_embedding_backward_workspace(uint64_t n, uint64_t rows, uint32_t dim) {
  if (n >= (1ull << 31) || rows > (1ull << 31)) return 0;
  return embed_grad_plan(n, rows, dim).bytes;
}

extern "C" ann_status ann_embedding_backward(const void *dy, uint64_t dy_stride, uint32_t type, const uint32_t *ids, uint64_t n, float scale,
                                             uint64_t rows, uint32_t dim, void *dtable, uint64_t dtable_stride, uint32_t table_type,
                                             uint32_t accumulate, void *workspace, uint64_t workspace_bytes, void *stream) {
  if (ann_status s = check_embedding("ann_embedding_backward", n, rows, dim, table_type, type)) return s;
  if ((n && (!dy || !ids)) || (rows && !dtable)) return fail(ANN_EINVAL, "ann_embedding_backward: NULL argument");
  if ((n && dy_stride < dim) || (rows && dtable_stride < dim)) return fail(ANN_EINVAL, "ann_embedding_backward: a row stride is shorter than a row");
  const EmbedGradPlan p = embed_grad_plan(n, rows, dim);
  if (p.bytes && !workspace) return fail(ANN_EINVAL, "ann_embedding_backward: workspace is NULL");
  if (workspace_bytes < p.bytes)
    return fail(ANN_EINVAL, "ann_embedding_backward: workspace of %llu bytes, %llu are needed", (unsigned long long)workspace_bytes,
                (unsigned long long)p.bytes);
  if (p.bytes && (uintptr_t)workspace % 16) return fail(ANN_EINVAL, "ann_embedding_backward: workspace is not aligned to 16 bytes");
  EmbedArgs g = {};
  g.from = dy, g.to = dtable, g.ids = ids, g.n = n, g.rows = rows, g.from_stride = dy_stride, g.to_stride = dtable_stride, g.dim = dim, g.scale = scale;
  g.accumulate = accumulate;
  char *ws = (char *)workspace;
  const hipStream_t st = (hipStream_t)stream;
  if (type == ANN_F32) return embedding_backward<float, float>(p, g, ws, st);
  if (type == ANN_F16) return table_type == ANN_F32 ? embedding_backward<f16_t, float>(p, g, ws, st) : embedding_backward<f16_t, f16_t>(p, g, ws, st);
  return table_type == ANN_F32 ? embedding_backward<bf16_t, float>(p, g, ws, st) : embedding_backward<bf16_t, bf16_t>(p, g, ws, st);
}
