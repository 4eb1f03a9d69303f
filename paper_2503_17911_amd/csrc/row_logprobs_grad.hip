// Gradients of the rows' log probabilities and of the softmax' entropy.
//
//   G[i][j] = g_i ([j = t_i] - p_ij) - h_i p_ij (s_ij - lse_i + H_i),  p_ij = exp(s_ij - lse_i)
//   dq = scale G X,  dX = scale G^T Q,  dbias_j = sum_i G_ij
//
// A chunk of rows at a time: G of the chunk from the scores' product once more
// (G in 16 bits, or fp32 with fp32 rows; at most kChunkBytes of it), then its two
// products.  Sums over the rows (dq) are kept in fp32 from chunk to chunk, shared
// out over the workgroups and joined in a fixed order; those over the queries (dX)
// are whole within a chunk.
//
// G in 16 bits: bf16 has the range for any probability.  f16 does not (a million
// like rows have p = 2^-20, its smallest normal number is 2^-14), so G is stored
// times the power of two that brings |g| + |h| (H + 1/e), which no element of G exceeds, to
// 2^13 .. 2^14; what lies 2^-28 below the largest then starts to lose bits, 2^-38 is
// lost, which a sum over 2^31 rows cannot show in f16.  The element of the given row
// is formed as g (1 - p) in fp32 before it is rounded: apart, g x_t and g p x_t would cancel.
// What its rounding leaves goes to dq in fp32: that element outweighs all others
// and rows of a cluster are alike, so that dq, their difference, erred by 0.6 % (bf16) with it, 0.17 % is the rounding of dq.
#include "row_logprobs.hpp"

#include <math.h>

namespace ann {

constexpr uint64_t kChunkBytes = 512ull << 20;  // of G at a time
constexpr uint32_t kGradTarget = 768;           // workgroups of a product: three to a compute unit

struct GradArgs {
  ScoreTable g;
  const uint32_t *targets;
  const float *lse, *entropy, *g_logprob, *g_entropy;
  const float *scaling;  // [2]: what G is multiplied by before it is rounded, and its inverse (f16)
  float *rest;           // [nq]: what the rounding of the given row's element left (16 bits)
};

// scaling[0]: the power of two for G, scaling[1]: its inverse.
__global__ __launch_bounds__(1024) void grad_scaling_kernel(GradArgs a, float *__restrict__ scaling) {
  __shared__ float room[16];
  float most = 0.0f;
  for (uint32_t i = threadIdx.x; i < a.g.nq; i += 1024) {
    float v = a.g_logprob ? fabsf(a.g_logprob[i]) : 0.0f;
    if (a.g_entropy) v += fabsf(a.g_entropy[i]) * (fabsf(a.entropy[i]) + 0.375f);
    most = fmaxf(most, v);
  }
  most = wave_max_f32(most);
  if (threadIdx.x % kWave == 0) room[threadIdx.x / kWave] = most;
  __syncthreads();
  if (threadIdx.x != 0) return;
  for (int w = 0; w < 16; ++w) most = fmaxf(most, room[w]);
  int e = 0;
  if (most > 0.0f && most < INFINITY) frexpf(most, &e);  // most < 2^e
  e = e < -100 ? -100 : e > 100 ? 100 : e;
  scaling[0] = ldexpf(1.0f, 14 - e);
  scaling[1] = ldexpf(1.0f, e - 14);
}

// G of rows row0 .. row0 + rows (of this chunk), [nq][ld], zero from row n on.  m runs over rows, n over queries, so that a lane holds runs of
// four rows of one query.  BIAS: biases and rows left out.  SUMS: row_sums[2 q_tile + half][ld] gets sums over 64 queries.
template <typename T, bool BIAS, bool ENTROPY, bool SUMS>
__global__ __launch_bounds__(256) void grad_scores_kernel(GradArgs a, uint32_t row0, uint32_t q_tiles, uint32_t ld, T *__restrict__ G,
                                                          float *__restrict__ row_sums) {
  __shared__ __attribute__((aligned(16))) char lds[kTileBytes<T, kAlong, kAlong>];
  __shared__ float row_bias[kTile];
  const ScoreTable &g = a.g;
  // a die takes a row tile through all queries
  const uint32_t row_tiles = ld / kTile, qt = blockIdx.x / 8 % q_tiles, rt = blockIdx.x / 8 / q_tiles * 8 + blockIdx.x % 8;
  if (rt >= row_tiles) return;
  const int wave = (int)threadIdx.x / kWave, lane = lane_id(), mw = wave / 2 * 64, nw = wave % 2 * 64;
  const Lines<T> X = {(const T *)g.rows, g.row_stride, g.n, g.d}, Q = {(const T *)g.q, g.q_stride, g.nq, g.d};
  const uint32_t first = row0 + rt * kTile;
  if (threadIdx.x < kTile) row_bias[threadIdx.x] = first + threadIdx.x < g.n ? (BIAS ? g.bias[first + threadIdx.x] : 0.0f) : -INFINITY;
  f32x16 acc[2][2];
  clear(acc);
  tile_product<T, kAlong, kAlong>(acc, X, first, Q, qt * kTile, 0, g.d, lds);  // (its barriers stand between row_bias and its use)
  const bool whole = first + kTile <= g.n;
  const float scaling = sizeof(T) == 2 && a.scaling ? a.scaling[0] : 1.0f;
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const uint32_t q = qt * kTile + nw + j * 32 + lane % 32;
    const bool there = q < g.nq;
    const uint32_t target = there && a.targets ? a.targets[q] : ANN_PAD_ID;
    float lse = there ? a.lse[q] : 0.0f;
    const bool none = !there || lse == -INFINITY;
    if (none) lse = 0.0f;
    const float gl = none || !a.g_logprob || target >= g.n ? 0.0f : a.g_logprob[q];
    const float gh = ENTROPY && !none ? a.g_entropy[q] : 0.0f, h = ENTROPY && !none ? a.entropy[q] : 0.0f;
    const uint32_t hit = target - (first + mw);  // row of the target within the wavefront's 64, if below 64
#pragma unroll
    for (int i = 0; i < 2; ++i) {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        float s = acc[i][j][r], bias = 0.0f;
        if (BIAS || !whole) bias = row_bias[mw + i * 32 + block_row(r)];
        s = __builtin_fmaf(s, g.scale, bias) - lse;
        const float p = __builtin_amdgcn_exp2f(s * kLog2e);
        const float slope = ENTROPY ? __builtin_fmaf(gh, s + h, gl) : gl;
        float v = -(p * slope);
        if ((uint32_t)(i * 32 + block_row(r)) == hit) v += gl;
        if ((BIAS || !whole) && bias == -INFINITY) v = 0.0f;
        acc[i][j][r] = none ? 0.0f : v;
      }
      if (there) {
        T *out = G + (uint64_t)q * ld + rt * kTile + mw + i * 32 + lane / 32 * 4;
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
          Piece<T, 4> o;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            o.v[e] = from_f32<T>(acc[i][j][r + e] * scaling);
            if (sizeof(T) == 2 && (uint32_t)(i * 32 + block_row(r + e)) == hit) a.rest[q] = __builtin_fmaf(acc[i][j][r + e], scaling, -to_f32(o.v[e]));
          }
          *(Piece<T, 4> *)(out + r * 2) = o;
        }
      }
    }
  }
  if constexpr (SUMS) {
    float mine = 0.0f;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        float v = acc[i][0][r] + acc[i][1][r];
        v += __int_as_float(dpp_i32<kDppQuadXor1>(__float_as_int(v)));
        v += __int_as_float(dpp_i32<kDppQuadXor2>(__float_as_int(v)));
        v += __int_as_float(dpp_i32<kDppRowHalfMirror>(__float_as_int(v)));
        v += __int_as_float(dpp_i32<kDppRowMirror>(__float_as_int(v)));
        const LanePair p = lane_pair<true>(__float_as_uint(v));
        v = __uint_as_float(p.low) + __uint_as_float(p.high);
        if (lane % 32 == i * 16 + r) mine = v;
      }
    const int i = lane % 32 / 16, r = lane % 16;
    row_sums[(uint64_t)(qt * 2 + wave % 2) * ld + rt * kTile + mw + i * 32 + block_row(r)] = mine;
  }
}

// part[split][q][c] (+)= sum over the split's rows of the chunk of G[q][j] x[j][c]  (rows left out may hold anything: read as zeros)
template <typename T>
__global__ __launch_bounds__(256) void grad_queries_kernel(ScoreTable g, uint32_t row0, uint32_t rows, uint32_t ld, const T *__restrict__ G, uint32_t splits,
                                                           float *__restrict__ part, bool add) {
  __shared__ __attribute__((aligned(16))) char lds[kTileBytes<T, kAlong, kAcross>];
  const uint32_t c_tiles = (g.d + kTile - 1) / kTile, q_tiles = (g.nq + kTile - 1) / kTile;
  const uint32_t ct = blockIdx.x % c_tiles, qt = blockIdx.x / c_tiles % q_tiles, split = blockIdx.x / c_tiles / q_tiles;
  const uint32_t slices = (rows + Operand16<T>::kSlice - 1) / Operand16<T>::kSlice;
  const uint32_t begin = (uint32_t)((uint64_t)slices * split / splits) * Operand16<T>::kSlice;
  uint32_t end = (uint32_t)((uint64_t)slices * (split + 1) / splits) * Operand16<T>::kSlice;
  if (end > rows) end = rows;
  const Lines<T> A = {G, ld, g.nq, rows}, B = {(const T *)g.rows + row0 * g.row_stride, g.row_stride, g.d, rows, g.bias ? g.bias + row0 : nullptr};
  f32x16 acc[2][2];
  clear(acc);
  tile_product<T, kAlong, kAcross>(acc, A, qt * kTile, B, ct * kTile, begin, end, lds);
  const int wave = (int)threadIdx.x / kWave, lane = lane_id();
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const uint32_t c = ct * kTile + wave % 2 * 64 + j * 32 + lane % 32;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const uint32_t q = qt * kTile + wave / 2 * 64 + i * 32 + block_row(r);
        if (q < g.nq && c < g.d) {
          float *p = part + ((uint64_t)split * g.nq + q) * g.d + c;
          *p = add ? *p + acc[i][j][r] : acc[i][j][r];
        }
      }
    }
}

// dq[q][c] = scale sum over the splits, in their order, and what was left of the given row's element
template <typename T>
__global__ __launch_bounds__(256) void grad_queries_sum_kernel(GradArgs a, const float *__restrict__ part, uint32_t splits, T *__restrict__ dq, uint64_t stride) {
  const ScoreTable &g = a.g;
  const uint64_t at = blockIdx.x * 256ull + threadIdx.x, all = (uint64_t)g.nq * g.d;
  if (at >= all) return;
  float sum = 0.0f;
  for (uint32_t s = 0; s < splits; ++s) sum += part[s * all + at];
  const uint64_t q = at / g.d, c = at % g.d;
  if (sizeof(T) == 2 && a.targets) {
    const uint32_t target = a.targets[q];
    if (target < g.n && !(g.bias && g.bias[target] == -INFINITY))
      sum = __builtin_fmaf(a.rest[q], to_f32(((const T *)g.rows)[target * g.row_stride + c]), sum);
  }
  dq[q * stride + c] = from_f32<T>(sum * (a.scaling ? g.scale * a.scaling[1] : g.scale));
}

// drows[row0 + j][c] = scale sum over the queries of G[q][j] q[q][c]
template <typename T>
__global__ __launch_bounds__(256) void grad_rows_kernel(ScoreTable g, uint32_t row0, uint32_t rows, uint32_t ld, const T *__restrict__ G, T *__restrict__ out,
                                                        uint64_t stride, const float *__restrict__ scaling) {
  __shared__ __attribute__((aligned(16))) char lds[kTileBytes<T, kAcross, kAcross>];
  const uint32_t c_tiles = (g.d + kTile - 1) / kTile, ct = blockIdx.x % c_tiles, rt = blockIdx.x / c_tiles;
  const Lines<T> A = {G, ld, ld, g.nq}, B = {(const T *)g.q, g.q_stride, g.d, g.nq};
  f32x16 acc[2][2];
  clear(acc);
  tile_product<T, kAcross, kAcross>(acc, A, rt * kTile, B, ct * kTile, 0, g.nq, lds);
  const int wave = (int)threadIdx.x / kWave, lane = lane_id();
  const float by = scaling ? g.scale * scaling[1] : g.scale;
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const uint32_t c = ct * kTile + wave % 2 * 64 + j * 32 + lane % 32;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const uint32_t row = rt * kTile + wave / 2 * 64 + i * 32 + block_row(r);
        if (row < rows && c < g.d) {
          const bool left_out = g.bias && g.bias[row0 + row] == -INFINITY;  // (zero, whatever the queries hold)
          out[(uint64_t)(row0 + row) * stride + c] = from_f32<T>(left_out ? 0.0f : acc[i][j][r] * by);
        }
      }
    }
}

// drow_bias[row0 + j] = sum of the parts, in their order
__global__ __launch_bounds__(256) void grad_bias_kernel(const float *__restrict__ row_sums, uint32_t parts, uint32_t ld, uint32_t row0, uint32_t rows,
                                                        float *__restrict__ out) {
  const uint32_t j = blockIdx.x * 256 + threadIdx.x;
  if (j >= rows) return;
  float sum = 0.0f;
  for (uint32_t p = 0; p < parts; ++p) sum += row_sums[(uint64_t)p * ld + j];
  out[row0 + j] = sum;
}

// ---------------------------------------------------------------------------
struct BackwardPlan {
  uint32_t q_tiles = 0, chunk = 0, splits = 0;  // chunk: rows at a time, a multiple of kTile
  uint64_t g_at = 0, part_at = 0, sums_at = 0, scaling_at = 0, rest_at = 0;
  Parts parts;
};

static BackwardPlan backward_plan(uint32_t nq, uint64_t n, uint32_t d, uint32_t type) {
  BackwardPlan p;
  if (nq == 0 || n == 0) return p;
  p.q_tiles = (nq + kTile - 1) / kTile;
  const uint64_t row_bytes = (uint64_t)nq * type_bytes(type), all = (n + kTile - 1) / kTile * kTile;
  uint64_t chunk = kChunkBytes / row_bytes / kTile * kTile;
  if (chunk < kTile) chunk = kTile;
  if (chunk > all) chunk = all;
  // chunks of like sizes
  const uint64_t chunks = (all + chunk - 1) / chunk;
  p.chunk = (uint32_t)((all / kTile + chunks - 1) / chunks * kTile);
  const uint32_t tiles = p.q_tiles * ((d + kTile - 1) / kTile), most = (p.chunk + 511) / 512;
  p.splits = (kGradTarget + tiles - 1) / tiles;
  if (p.splits > most) p.splits = most;
  p.g_at = p.parts.take(p.chunk * row_bytes);
  p.part_at = p.parts.take((uint64_t)p.splits * nq * d * sizeof(float));
  p.sums_at = p.parts.take((uint64_t)p.q_tiles * 2 * p.chunk * sizeof(float));
  p.scaling_at = p.parts.take(2 * sizeof(float));
  p.rest_at = p.parts.take(nq * sizeof(float));
  return p;
}

struct GradOut {
  void *dq, *drows;
  float *drow_bias;
  uint64_t dq_stride, drows_stride;
};

template <typename T>
static ann_status backward(const GradArgs &args, const BackwardPlan &p, const GradOut &o, char *ws, hipStream_t st) {
  GradArgs a = args;
  const ScoreTable &g = a.g;
  const uint32_t c_tiles = (g.d + kTile - 1) / kTile;
  T *G = (T *)(ws + p.g_at);
  float *part = (float *)(ws + p.part_at), *sums = (float *)(ws + p.sums_at);
  a.rest = (float *)(ws + p.rest_at);
  if (sizeof(T) == 2 && std::is_same<T, f16_t>::value && g.nq && g.n) {
    float *scaling = (float *)(ws + p.scaling_at);
    grad_scaling_kernel<<<1, 1024, 0, st>>>(a, scaling);
    ANN_HIP(hipGetLastError());
    a.scaling = scaling;
  }
  // (no queries: one chunk of all rows, of which no product takes anything)
  const uint32_t chunk = p.chunk ? p.chunk : (g.n + kTile - 1) / kTile * kTile;
  for (uint32_t row0 = 0; row0 < g.n; row0 += chunk) {
    const uint32_t rows = g.n - row0 < chunk ? g.n - row0 : chunk, ld = (rows + kTile - 1) / kTile * kTile;
    if (g.nq) {
      const uint32_t grid = p.q_tiles * ((ld / kTile + 7) / 8 * 8);
      const auto run = [&](auto bias, auto entropy, auto row_sums) {
        grad_scores_kernel<T, decltype(bias)::value, decltype(entropy)::value, decltype(row_sums)::value><<<grid, 256, 0, st>>>(a, row0, p.q_tiles, ld, G, sums);
      };
      const auto run_sums = [&](auto bias, auto entropy) {
        if (o.drow_bias)
          run(bias, entropy, std::true_type());
        else
          run(bias, entropy, std::false_type());
      };
      const auto run_entropy = [&](auto bias) {
        if (a.g_entropy)
          run_sums(bias, std::true_type());
        else
          run_sums(bias, std::false_type());
      };
      if (g.bias)
        run_entropy(std::true_type());
      else
        run_entropy(std::false_type());
      ANN_HIP(hipGetLastError());
      if (o.dq) {
        grad_queries_kernel<T><<<c_tiles * p.q_tiles * p.splits, 256, 0, st>>>(g, row0, rows, ld, G, p.splits, part, row0 != 0);
        ANN_HIP(hipGetLastError());
      }
    }
    if (o.drows) {
      grad_rows_kernel<T><<<c_tiles * (ld / kTile), 256, 0, st>>>(g, row0, rows, ld, G, (T *)o.drows, o.drows_stride, a.scaling);
      ANN_HIP(hipGetLastError());
    }
    if (o.drow_bias) {
      grad_bias_kernel<<<(rows + 255) / 256, 256, 0, st>>>(sums, p.q_tiles * 2, ld, row0, rows, o.drow_bias);
      ANN_HIP(hipGetLastError());
    }
  }
  if (o.dq && g.nq) {
    const uint64_t all = (uint64_t)g.nq * g.d;
    grad_queries_sum_kernel<T><<<(uint32_t)((all + 255) / 256), 256, 0, st>>>(a, part, g.n ? p.splits : 0, (T *)o.dq, o.dq_stride);
    ANN_HIP(hipGetLastError());
  }
  return ANN_OK;
}

}  // namespace ann

using namespace ann;

extern "C" uint64_t ann_row_logprobs_backward_workspace(uint32_t nq, uint64_t n, uint32_t d, uint32_t type) {
  if (n >= (1ull << 31) || nq >= (1u << 31) || d == 0 || type > ANN_BF16) return 0;
  return backward_plan(nq, n, d, type).parts.bytes;
}

extern "C" ann_status ann_row_logprobs_backward(const ann_row_scores *scores, const float *lse, const float *entropy, const float *g_logprob,
                                                const float *g_entropy, void *dq, uint64_t dq_stride, void *drows, uint64_t drows_stride,
                                                float *drow_bias, void *workspace, uint64_t workspace_bytes, void *stream) {
  if (ann_status s = check_scores("ann_row_logprobs_backward", scores)) return s;
  if (scores->nq && !lse) return fail(ANN_EINVAL, "ann_row_logprobs_backward: lse is NULL");
  if (scores->nq && g_entropy && !entropy) return fail(ANN_EINVAL, "ann_row_logprobs_backward: g_entropy without entropy");
  if (dq && dq_stride < scores->d) return fail(ANN_EINVAL, "ann_row_logprobs_backward: dq_stride is shorter than a row");
  if (drows && drows_stride < scores->d) return fail(ANN_EINVAL, "ann_row_logprobs_backward: drows_stride is shorter than a row");
  const BackwardPlan p = backward_plan(scores->nq, scores->n, scores->d, scores->type);
  if (ann_status s = check_workspace("ann_row_logprobs_backward", workspace, workspace_bytes, p.parts.bytes)) return s;
  GradArgs a = {};
  a.g = score_table(*scores);
  a.targets = scores->targets, a.lse = lse, a.entropy = entropy, a.g_logprob = g_logprob, a.g_entropy = g_entropy;
  const GradOut o = {dq, drows, drow_bias, dq_stride, drows_stride};
  if (scores->type == ANN_F32) return backward<float>(a, p, o, (char *)workspace, (hipStream_t)stream);
  if (scores->type == ANN_F16) return backward<f16_t>(a, p, o, (char *)workspace, (hipStream_t)stream);
  return backward<bf16_t>(a, p, o, (char *)workspace, (hipStream_t)stream);
}
