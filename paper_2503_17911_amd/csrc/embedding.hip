// Rows of a table by their ids, times a scale, and the table's gradient.
//
//   y[i] = scale * table[ids[i]];   dtable[r] = scale * sum over i with ids[i] = r of dy[i]
//
// Bound by memory.  Forward: a row belongs to 16 or 64 lanes, pieces of 16 bytes of the output with any alignment.  Gradient: the ids
// are put in order with their positions (id_sort), so that a table's row is a run of entries and its sum has a fixed order; no
// atomic that a result depends on.  Frequent ids make runs of any length, so runs do not go to lanes: a workgroup takes kChunk entries in
// order, sums them in fp32 and writes the runs that lie within; the ends of runs that cross a border go to the workspace, from where a
// second kernel joins them in the borders' order.  Rows without an id are filled with zeros beside the sums (a bit to a row
// says which; few ids: the whole table is filled beside the sorting).
#include "id_sort.hpp"
#include "row_pieces.hpp"

#include <type_traits>

namespace ann {

constexpr uint32_t kChunk = 32;           // entries that are summed one after the other
constexpr uint32_t kMostChunks = 1 << 15;  // beyond, chunks are longer
constexpr uint32_t kFetched = 8;          // rows on their way at a time

struct EmbedArgs {
  const void *from;  // forward: the table; backward: dy
  void *to;          // forward: y; backward: dtable
  const uint32_t *ids;
  uint64_t n, rows, from_stride, to_stride;
  uint32_t dim;
  float scale;
  // backward
  const uint32_t *keys, *positions, *hit;
  float *part;  // [chunks][2][dim]: the end of a run from the chunk before; the beginning of one that goes on in the next
  uint32_t chunk, chunks, accumulate;
};

// F: the table's type, T: of y
template <typename F, typename T, int LANES>
__global__ __launch_bounds__(256) void embed_kernel(EmbedArgs g) {
  constexpr int VEC = 16 / (int)sizeof(T), kGroups = 256 / LANES, kParts = VEC * (int)sizeof(F) / 16;
  const uint32_t lane = threadIdx.x % LANES;
  for (uint64_t i = (uint64_t)blockIdx.x * kGroups + threadIdx.x / LANES; i < g.n; i += (uint64_t)gridDim.x * kGroups) {
    const uint32_t id = g.ids[i];
    const bool there = id < g.rows;
    const F *from = (const F *)g.from + (there ? id : 0) * g.from_stride;
    T *to = (T *)g.to + i * g.to_stride;
    for (uint32_t c = lane * VEC; c < g.dim; c += LANES * VEC) {
      RowPiece<T, VEC> o;
      if (there) {
        RowPiece<F, VEC / kParts> v[kParts];
#pragma unroll
        for (int p = 0; p < kParts; ++p) v[p].load(from, c + p * (VEC / kParts), g.dim);
#pragma unroll
        for (int e = 0; e < VEC; ++e) o.v[e] = from_f32<T>(to_f32(v[e / (VEC / kParts)].v[e % (VEC / kParts)]) * g.scale);
      } else {
#pragma unroll
        for (int e = 0; e < VEC; ++e) o.v[e] = (T)0.0f;
      }
      o.store(to, c, g.dim);
    }
  }
}

// Rows of zeros; hit: but those whose bit is set.
template <typename F>
__global__ __launch_bounds__(256) void embed_zero_kernel(F *__restrict__ table, uint64_t rows, uint64_t stride, uint32_t dim, const uint32_t *__restrict__ hit) {
  constexpr int VEC = 16 / (int)sizeof(F);
  RowPiece<F, VEC> zero;
#pragma unroll
  for (int e = 0; e < VEC; ++e) zero.v[e] = (F)0.0f;
  for (uint64_t r = (uint64_t)blockIdx.x * 4 + threadIdx.x / 64; r < rows; r += (uint64_t)gridDim.x * 4) {
    if (hit && hit[r / 32] >> (r % 32) & 1) continue;
    for (uint32_t c = threadIdx.x % 64 * VEC; c < dim; c += 64 * VEC) zero.store(table + r * stride, c, dim);
  }
}

template <typename F, int VEC>
__device__ __forceinline__ void write_gradient(const EmbedArgs &g, uint32_t row, uint32_t c, const float (&sum)[VEC]) {
  F *to = (F *)g.to + row * g.to_stride;
#pragma unroll
  for (int e = 0; e < VEC; ++e) {
    if (c + e >= g.dim) break;
    const float old = g.accumulate ? to_f32(to[c + e]) : 0.0f;
    to[c + e] = from_f32<F>(g.accumulate ? __builtin_fmaf(sum[e], g.scale, old) : sum[e] * g.scale);
  }
}

// T: of dy, F: of the table.  A group of LANES lanes takes a chunk and LANES * VEC columns.
template <typename T, typename F, int LANES>
__global__ __launch_bounds__(256) void embed_grad_kernel(EmbedArgs g) {
  constexpr int VEC = 16 / (int)sizeof(T), kGroups = 256 / LANES;
  const uint32_t tiles = (g.dim + LANES * VEC - 1) / (LANES * VEC);
  const uint64_t at = (uint64_t)blockIdx.x * kGroups + threadIdx.x / LANES;
  const uint64_t chunk = at / tiles;
  const uint32_t c = ((uint32_t)(at % tiles) * LANES + threadIdx.x % LANES) * VEC;
  if (chunk >= g.chunks) return;
  const uint64_t begin = chunk * g.chunk, end = begin + g.chunk < g.n ? begin + g.chunk : g.n;
  uint32_t row = g.keys[begin];
  bool first = begin != 0 && g.keys[begin - 1] == row;  // the run began before this chunk
  const uint32_t next = end < g.n ? g.keys[end] : 0xFFFFFFFFu;
  float sum[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) sum[e] = 0.0f;
  const auto finish = [&](bool goes_on) {
    if (row >= g.rows || c >= g.dim) return;
    if (first || goes_on) {
      float *to = g.part + (chunk * 2 + (first ? 0 : 1)) * g.dim + c;
#pragma unroll
      for (int e = 0; e < VEC; ++e)
        if (c + e < g.dim) to[e] = sum[e];
    } else {
      write_gradient<F, VEC>(g, row, c, sum);
    }
  };
  for (uint64_t i0 = begin; i0 < end; i0 += kFetched) {
    RowPiece<T, VEC> v[kFetched];
    uint32_t key[kFetched];
#pragma unroll
    for (uint32_t u = 0; u < kFetched; ++u) {
      const uint64_t i = i0 + u < end ? i0 + u : end - 1;
      key[u] = g.keys[i];
      if (key[u] < g.rows) v[u].load((const T *)g.from + g.positions[i] * g.from_stride, c, g.dim);
    }
#pragma unroll
    for (uint32_t u = 0; u < kFetched; ++u) {
      if (i0 + u >= end || key[u] >= g.rows) continue;  // (what belongs to no row comes last)
      if (key[u] != row) {
        finish(false);
        row = key[u], first = false;
#pragma unroll
        for (int e = 0; e < VEC; ++e) sum[e] = 0.0f;
      }
#pragma unroll
      for (int e = 0; e < VEC; ++e) sum[e] += to_f32(v[u].v[e]);
    }
  }
  finish(row == next);
}

// Runs that cross borders between chunks, by the chunk in which they begin.  64 columns to a workgroup of four wavefronts, a run of the chunks to each.
template <typename F>
__global__ __launch_bounds__(256) void embed_join_kernel(EmbedArgs g) {
  __shared__ float room[4][64];
  const uint64_t chunk = blockIdx.x;
  const uint64_t border = (chunk + 1) * g.chunk;
  if (border >= g.n) return;
  const uint32_t row = g.keys[border];
  if (row >= g.rows || g.keys[border - 1] != row) return;
  // (the run begins in this chunk: at its first entry at the earliest)
  const uint64_t begin = chunk * g.chunk;
  if (begin != 0 && g.keys[begin - 1] == row) return;
  // the chunks after this one that begin with it
  const uint32_t lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  uint64_t last = chunk + 1;
  for (;;) {
    const uint64_t next = last + 1 + lane;
    const uint64_t mine = __ballot(next < g.chunks && g.keys[next * g.chunk] == row);
    last += __builtin_ctzll(~mine | (mine == ~0ull ? 1ull : 0ull)) + (mine == ~0ull ? 64 : 0);
    if (mine != ~0ull) break;
  }
  const uint64_t count = last - chunk, from = chunk + 1 + count * wave / 4, to = chunk + 1 + count * (wave + 1) / 4;
  for (uint32_t c0 = 0; c0 < g.dim; c0 += 64) {
    const uint32_t c = c0 + lane;
    float sum = 0.0f;
    if (c < g.dim) {
      if (wave == 0) sum = g.part[(chunk * 2 + 1) * g.dim + c];
      for (uint64_t k = from; k < to; k += 8) {
        float v[8];
#pragma unroll
        for (uint32_t u = 0; u < 8; ++u) v[u] = k + u < to ? g.part[(k + u) * 2 * g.dim + c] : 0.0f;
#pragma unroll
        for (uint32_t u = 0; u < 8; ++u) sum += v[u];
      }
    }
    __syncthreads();
    room[wave][lane] = sum;
    __syncthreads();
    if (wave == 0 && c < g.dim) {
      const float total[1] = {((sum + room[1][lane]) + room[2][lane]) + room[3][lane]};
      write_gradient<F, 1>(g, row, c, total);
    }
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
  p.chunk = kChunk;
  while ((n + p.chunk - 1) / p.chunk > kMostChunks) p.chunk *= 2;
  p.chunks = (uint32_t)((n + p.chunk - 1) / p.chunk);
  p.part_at = p.sort.bytes;
  p.hit_at = p.part_at + ((uint64_t)p.chunks * 2 * dim * sizeof(float) + 255) / 256 * 256;
  p.bytes = p.hit_at + ((rows + 31) / 32 * 4 + 255) / 256 * 256;
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
  uint32_t *hit = (uint32_t *)(ws + p.hit_at);
  const uint32_t zero_blocks = (uint32_t)((g.rows + 3) / 4 < 4096 ? (g.rows + 3) / 4 : 4096);
  const bool small = g.n <= kSmallSort;
  // (few ids: all rows, before anything else is written)
  if (!g.accumulate && g.rows && small) {
    embed_zero_kernel<F><<<zero_blocks, 256, 0, st>>>((F *)g.to, g.rows, g.to_stride, g.dim, nullptr);
    ANN_HIP(hipGetLastError());
  }
  if (g.n == 0 || g.rows == 0) return ANN_OK;
  SortedIds sorted;
  if (ann_status s = sort_ids(p.sort, g.ids, ws, small || g.accumulate ? nullptr : hit, st, sorted)) return s;
  if (!g.accumulate && !small) {
    embed_zero_kernel<F><<<zero_blocks, 256, 0, st>>>((F *)g.to, g.rows, g.to_stride, g.dim, hit);
    ANN_HIP(hipGetLastError());
  }
  g.keys = sorted.keys, g.positions = sorted.positions, g.part = (float *)(ws + p.part_at), g.chunk = p.chunk, g.chunks = p.chunks;
  constexpr uint32_t VEC = 16 / sizeof(T);
  const auto sums = [&](auto lanes) {
    constexpr uint32_t L = decltype(lanes)::value;
    const uint64_t groups = (uint64_t)p.chunks * ((g.dim + L * VEC - 1) / (L * VEC));
    embed_grad_kernel<T, F, L><<<(uint32_t)((groups * L + 255) / 256), 256, 0, st>>>(g);
  };
  if (g.dim <= 16 * VEC)
    sums(std::integral_constant<int, 16>());
  else
    sums(std::integral_constant<int, 64>());
  ANN_HIP(hipGetLastError());
  if (p.chunks > 1) {
    embed_join_kernel<F><<<p.chunks - 1, 256, 0, st>>>(g);
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
    constexpr uint32_t VEC = 16 / sizeof(T);
    const uint32_t lanes = dim <= 16 * VEC ? 16 : 64;
    const uint64_t want = (n * lanes + 255) / 256;
    const uint32_t blocks = (uint32_t)(want < 16384 ? want : 16384);
    if (lanes == 16)
      embed_kernel<F, T, 16><<<blocks, 256, 0, st>>>(g);
    else
      embed_kernel<F, T, 64><<<blocks, 256, 0, st>>>(g);
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
