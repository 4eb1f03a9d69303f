// Rows of a table by their ids, times a scale, and the table's gradient.
//
//   y[i] = scale * table[ids[i]];   dtable[r] = scale * sum over i with ids[i] = r of dy[i]
//
// Bound by memory.  Forward: a row belongs to 16, 32 or 64 lanes, pieces of 16 bytes of the output with any alignment.  Gradient: the ids
// are put in order with their positions (id_sort.hpp), so that a table's row is the sum of a run of entries (row_runs.hpp).  Rows without an id are filled
// with zeros beside the sorting, which leaves most of the card idle: with few ids the whole table, with many what the first pass over the ids found no id for.
// Measured: 80,000 x 960 fp32 to bf16 57 us (246 MB of distinct rows and output; frequent rows are read into each die's L2); gradient of 80,000 x 768 bf16 into
// 50,000 fp32 rows 98 us: order 34 with the zeros beside it, runs 45 to 47, their join 10; of 5,003 x 100 fp16 22 us.
#include "row_runs.hpp"

namespace ann {

constexpr uint64_t kPastBytes = 64ull << 20;  // outputs larger than this are stored past the caches (80,000 x 960 bf16: 66 -> 59 us; a small one is read next)

struct EmbedArgs {
  const void *from;  // forward: the table; backward: dy
  void *to;          // forward: y; backward: dtable
  const uint32_t *ids;
  uint64_t n, rows, from_stride, to_stride;
  uint32_t dim, accumulate;
  float scale;
};

// F: the table's type, T: of y.  A group of LANES lanes takes kUnits pieces to a lane at a time, `slots` of them to a row: so many reads are on
// their way at once (80,000 x 960 fp32 to bf16: 98 us one after the other, 66 by four, 57 by eight and stored past the caches).
template <typename F, typename T, int LANES, RowEnd END>
__global__ __launch_bounds__(256) void embed_kernel(EmbedArgs g, uint32_t slots, bool past) {
  constexpr int VEC = 16 / (int)sizeof(T), kGroups = 256 / LANES, kParts = VEC * (int)sizeof(F) / 16, kEach = VEC / kParts, kUnits = 8;
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
      if (past)
        o.store_past((T *)g.to + row[u] * g.to_stride, c[u], g.dim);
      else
        o.store((T *)g.to + row[u] * g.to_stride, c[u], g.dim);
    }
  }
}

// Rows first .. end - 1 of zeros; hit: but those that it marks.
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
// pass' counting, the others beside its placing.  Two fifths, as the two take 4.5 and 8 to 9 us by themselves for 80,000 ids; it matters little: by one, two and
// three fifths 87.9, 87.0 and 89.2 us for 80,000 x 768 into 50,000 rows, 189, 186 and 186 into 200,000, 91, 90 and 88 for 200,000 x 128 into 200,000.
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

// What the sums of dy over runs of equal ids are and where they go.  T: of dy, F: of the table.
template <typename T, typename F>
struct TableGradient {
  static constexpr bool kWeighted = false, kScalar = false;
  const T *dy;
  F *table;
  const uint8_t *hit;
  uint64_t dy_stride, stride, rows;
  uint32_t dim, accumulate;
  float scale;
  __device__ __forceinline__ const T *row(uint32_t position) const { return dy + position * dy_stride; }
  __device__ __forceinline__ float weight(uint32_t) const { return 1.0f; }
  __device__ __forceinline__ float scalar(uint32_t) const { return 0.0f; }
  __device__ __forceinline__ void write_scalar(uint32_t, uint32_t, float) const {}
  __device__ __forceinline__ void beside(uint32_t block, uint32_t blocks) const { zero_rows<F>(table, 0, rows, stride, dim, hit, block, blocks); }
  template <int VEC, RowEnd END>
  __device__ __forceinline__ void write(uint32_t id, uint32_t, uint32_t c, const float (&sum)[VEC]) const {
    F *to = table + id * stride;
    if constexpr (VEC == 1) {
      to[c] = from_f32<F>(accumulate ? __builtin_fmaf(sum[0], scale, to_f32(to[c])) : sum[0] * scale);
    } else {
      constexpr int kEach = 16 / (int)sizeof(F), N = VEC < kEach ? VEC : kEach;
#pragma unroll
      for (int p = 0; p < VEC; p += N) {
        // (a piece at the row's end is read element by element: what another lane writes is not read)
        RowPiece<F, N, END == kWholePieces ? kWholePieces : kByElement> o;
        float v[N];
        if (accumulate) o.load(to, c + p, dim);
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = accumulate ? __builtin_fmaf(sum[p + e], scale, o.get(e)) : sum[p + e] * scale;
        o.set(v);
        o.store(to, c + p, dim);
      }
    }
  }
};

struct EmbedGradPlan {
  IdSortPlan sort;
  RunsPlan runs;
  uint64_t part_at = 0, hit_at = 0, bytes = 0;
};

static EmbedGradPlan embed_grad_plan(uint64_t n, uint64_t rows, uint32_t dim) {
  EmbedGradPlan p;
  if (n == 0) return p;
  p.sort = id_sort_plan(n, rows);
  p.runs = runs_plan(n, dim);
  p.part_at = p.sort.bytes;
  p.hit_at = p.part_at + p.runs.part_bytes;
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
  const Runs runs = {sorted.keys, sorted.positions, (uint32_t)g.n, (uint32_t)g.rows, p.runs.chunk, p.runs.chunks, g.dim, (float *)(ws + p.part_at), g.dim};
  const TableGradient<T, F> work = {(const T *)g.from, (F *)g.to, hit, g.from_stride, g.to_stride, g.rows, g.dim, g.accumulate, g.scale};
  return sum_runs<T>(runs, work, fill ? zero_blocks : 0, st);
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
      const uint64_t groups = (n * slots + 7) / 8, want = (groups * L + 255) / 256;
      embed_kernel<F, T, L, decltype(end)::value><<<(uint32_t)(want < 65536 ? want : 65536), 256, 0, st>>>(g, slots, n * dim * sizeof(T) > kPastBytes);
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
