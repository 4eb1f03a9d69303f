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
// 2^13 .. 2^14 for the query with the largest; what lies 2^-28 below that starts to lose bits, 2^-38 is
// lost: n such elements are less than half a step of the largest in f16 (2^-11 of it) up to n = 2^27, and queries
// with much smaller weights than the largest keep the bits that this leaves them.  The element of the given row
// is formed as g (1 - p) in fp32 before it is rounded: apart, g x_t and g p x_t would cancel.
// What its rounding leaves goes to dq in fp32: that element outweighs all others
// and rows of a cluster are alike, so that dq, their difference, erred by 0.6 % (bf16) with it, 0.17 % is the rounding of dq.
// The rows' gradient has few terms that count, often the given row's one alone: G's rounding would add to the result's (0.24 % instead of
// 0.17 % in bf16).  So what it leaves is taken along: where queries are few (kFewQueries) of every element, in 16 bits more, otherwise of the
// given rows' elements.  Where no given row's element outweighs the others (the entropy's gradient alone) G's rounding stays in the
// results: up to 0.20 % in dq and 0.22 % in the rows' gradient in bf16, 2.4e-4 and 2.9e-4 in f16.
#include "row_logprobs.hpp"

#include <math.h>

namespace ann {

constexpr uint64_t kChunkBytes = 512ull << 20;  // of G at a time
constexpr uint32_t kGradTarget = 768;           // workgroups of a product: three to a compute unit
constexpr uint32_t kWideSlots = 512;            // of a wide one: two

// Wavefronts to a SIMD of the gradients' products by tiles of 128 (three instead of two: 303 -> 237 and 282 -> 255 us with 2,048 x 50,000 x 768).
template <typename T>
constexpr int kGradWaves = sizeof(T) == 2 ? 3 : 2;

constexpr uint32_t kFewQueries = 256;  // up to so many, the rows' gradient takes all of G's remainders

struct GradArgs {
  ScoreTable g;
  const uint32_t *targets;
  const float *lse, *entropy, *g_logprob, *g_entropy;
  const float *scaling;  // [2]: what G is multiplied by before it is rounded, and its inverse (f16)
  float *rest;           // [nq]: what the rounding of the given row's element left (16 bits)
};

// scaling[0]: the power of two for G, scaling[1]: its inverse.  A query counts as it does in G: with g_logprob where a row is given, not at
// all without a row left (or with statistics that are NaN).  Weights that are not finite spoil their own query, not the scale of the others.
__global__ __launch_bounds__(1024) void grad_scaling_kernel(GradArgs a, float *__restrict__ scaling) {
  __shared__ float room[16];
  float most = 0.0f;
  for (uint32_t i = threadIdx.x; i < a.g.nq; i += 1024) {
    if (!(a.lse[i] > -INFINITY)) continue;
    const bool given = a.targets && a.targets[i] < a.g.n;
    const float g = a.g_logprob && given ? fabsf(a.g_logprob[i]) : 0.0f;
    const float h = a.g_entropy ? fabsf(a.g_entropy[i]) * (fabsf(a.entropy[i]) + 0.375f) : 0.0f;
    if (g < INFINITY && h < INFINITY) most = fmaxf(most, fminf(g + h, 3.402823466e38f));
  }
  most = wave_max_f32(most);
  if (threadIdx.x % kWave == 0) room[threadIdx.x / kWave] = most;
  __syncthreads();
  if (threadIdx.x != 0) return;
  for (int w = 0; w < 16; ++w) most = fmaxf(most, room[w]);
  int e = 0;
  if (most > 0.0f) frexpf(most, &e);  // most < 2^e, e <= 128
  e = e < -100 ? -100 : e;
  scaling[0] = ldexpf(1.0f, 14 - e);
  scaling[1] = ldexpf(1.0f, e - 14);
}

// G of rows row0 .. row0 + rows (of this chunk), [nq][ld], zero from row n on.  m runs over rows, n over queries, so that a lane holds runs of
// four rows of one query.  BIAS: biases and rows left out.  SUMS: row_sums[2 q_tile + half][ld] gets sums over 64 queries.
template <typename T, bool BIAS, bool ENTROPY, bool SUMS>
__global__ __launch_bounds__(256) void grad_scores_kernel(GradArgs a, uint32_t row0, uint32_t q_tiles, uint32_t ld, T *__restrict__ G,
                                                          T *__restrict__ rests, float *__restrict__ row_sums) {
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
  tile_product<T, kAlong, kAlong, sizeof(T) == 4>(acc, X, first, Q, qt * kTile, 0, g.d, lds);  // (its barriers stand between row_bias and its use)
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
        // (no probability: 0, also where the score is so low that its slope overflows)
        if (ENTROPY && !(p != 0.0f)) v = 0.0f;
        if ((uint32_t)(i * 32 + block_row(r)) == hit) v += gl;
        if ((BIAS || !whole) && bias == -INFINITY) v = 0.0f;
        acc[i][j][r] = none ? 0.0f : v;
      }
      if (there) {
        T *out = G + (uint64_t)q * ld + rt * kTile + mw + i * 32 + lane / 32 * 4;
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
          Piece<T, 4> o, left;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            o.v[e] = from_f32<T>(acc[i][j][r + e] * scaling);
            if (sizeof(T) == 2 && rests) left.v[e] = from_f32<T>(__builtin_fmaf(acc[i][j][r + e], scaling, -to_f32(o.v[e])));
            if (sizeof(T) == 2 && (uint32_t)(i * 32 + block_row(r + e)) == hit) a.rest[q] = __builtin_fmaf(acc[i][j][r + e], scaling, -to_f32(o.v[e]));
          }
          *(Piece<T, 4> *)(out + r * 2) = o;
          if (sizeof(T) == 2 && rests) *(Piece<T, 4> *)(rests + (out - G) + r * 2) = left;
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

// part[split][q][c] (+)= sum over the split's rows of the chunk of G[q][j] x[j][c]  (rows left out may hold anything: read as zeros, or,
// MB == 4, there are none)
// MB == 4: tiles of 256 queries by the wide product (2,048 x 50,000 x 768 fp16: 183 us, 860 TFLOP/s; by tiles of 128: 240).
template <typename T, int MB>
__global__ __launch_bounds__(256, MB == 4 ? 2 : kGradWaves<T>) void grad_queries_kernel(ScoreTable g, uint32_t row0, uint32_t rows, uint32_t ld, const T *__restrict__ G,
                                                                                        uint32_t splits, float *__restrict__ part, bool add) {
  constexpr int kQueryTile = MB * 64, kMore = MB == 4 ? kWideBuffer : 16, kSlice = MB == 4 ? kWideSlice : Operand16<T>::kSlice;
  __shared__ __attribute__((aligned(16))) char lds[MB == 4 ? kWideBuffer : kTileBytes<T, kAlong, kAcross>], lds1[kMore], lds2[kMore];
  const uint32_t c_tiles = (g.d + kTile - 1) / kTile, q_tiles = (g.nq + kQueryTile - 1) / kQueryTile;
  // workgroup b runs on die b mod 8: a die takes a run of rows through all columns and queries
  const uint32_t all = c_tiles * q_tiles * splits, per_die = (all + 7) / 8, in_die = blockIdx.x / 8, at = blockIdx.x % 8 * per_die + in_die;
  const uint32_t ct = at % c_tiles, qt = at / c_tiles % q_tiles, split = at / c_tiles / q_tiles;
  if (in_die >= per_die || at >= all) return;
  const uint32_t slices = (rows + kSlice - 1) / kSlice;
  const uint32_t begin = (uint32_t)((uint64_t)slices * split / splits) * kSlice;
  uint32_t end = (uint32_t)((uint64_t)slices * (split + 1) / splits) * kSlice;
  f32x16 acc[MB][2];
  clear(acc);
  if constexpr (MB == 4) {
    // (G is zero behind the last row)
    const Lines<T> A = {G, ld, g.nq, ld}, B = {(const T *)g.rows + row0 * g.row_stride, g.row_stride, g.d, rows};
    wide_product<T, kAlong, kAcross>(acc, A, qt * kQueryTile, B, ct * kTile, begin, end, lds, lds1, lds2);
  } else {
    if (end > rows) end = rows;
    const Lines<T> A = {G, ld, g.nq, rows}, B = {(const T *)g.rows + row0 * g.row_stride, g.row_stride, g.d, rows, g.bias ? g.bias + row0 : nullptr};
    tile_product<T, kAlong, kAcross>(acc, A, qt * kQueryTile, B, ct * kTile, begin, end, lds);
  }
  const int wave = (int)threadIdx.x / kWave, lane = lane_id();
#pragma unroll
  for (int i = 0; i < MB; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const uint32_t c = ct * kTile + wave % 2 * 64 + j * 32 + lane % 32;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const uint32_t q = qt * kQueryTile + wave / 2 * MB * 32 + i * 32 + block_row(r);
        if (q < g.nq && c < g.d) {
          float *p = part + ((uint64_t)split * g.nq + q) * g.d + c;
          *p = add ? *p + acc[i][j][r] : acc[i][j][r];
        }
      }
    }
}

// dq[q][c] = scale sum over the splits, and what was left of the given row's element.  A workgroup of THREADS lanes takes one
// query after LANES * RUNS of them: LANES to its columns, RUNS to runs of its splits, which are added in the runs' order.
// Eight splits' parts are on their way at a time.
template <typename T, int LANES, int RUNS, int THREADS>
__global__ __launch_bounds__(THREADS) void grad_queries_sum_kernel(GradArgs a, const float *__restrict__ part, uint32_t splits, T *__restrict__ dq, uint64_t stride) {
  constexpr int kQueries = THREADS / (LANES * RUNS);
  static_assert(RUNS == 1 || kQueries == 1, "runs are joined by the whole workgroup");
  __shared__ float room[RUNS > 1 ? RUNS : 1][RUNS > 1 ? LANES : 1];
  const ScoreTable &g = a.g;
  const uint64_t q = (uint64_t)blockIdx.x * kQueries + threadIdx.x / (LANES * RUNS), all = (uint64_t)g.nq * g.d;
  if (q >= g.nq) return;
  const float by = a.scaling ? g.scale * a.scaling[1] : g.scale;
  const uint32_t target = sizeof(T) == 2 && a.targets ? a.targets[q] : ANN_PAD_ID;
  const bool given = target < g.n && !(g.bias && g.bias[target] == -INFINITY);
  const float rest = given ? a.rest[q] : 0.0f;
  const uint32_t run = threadIdx.x / LANES % RUNS, end = (uint32_t)((uint64_t)splits * (run + 1) / RUNS);
  for (uint32_t c0 = 0; c0 < g.d; c0 += LANES) {
    const uint32_t c = c0 + threadIdx.x % LANES;
    float sum = 0.0f;
    if (c < g.d) {
      const float *p = part + q * g.d + c;
      uint32_t s = (uint32_t)((uint64_t)splits * run / RUNS);
      for (; s + 8 <= end; s += 8) {
        float v[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] = p[(s + u) * all];
#pragma unroll
        for (int u = 0; u < 8; ++u) sum += v[u];
      }
      for (; s < end; ++s) sum += p[s * all];
    }
    if constexpr (RUNS > 1) {
      __syncthreads();  // (the columns before have been read)
      room[run][threadIdx.x % LANES] = sum;
      __syncthreads();
      if (run != 0) continue;
#pragma unroll
      for (int r = 1; r < RUNS; ++r) sum += room[r][threadIdx.x % LANES];
    }
    if (c >= g.d) continue;
    if (given) sum = __builtin_fmaf(rest, to_f32(((const T *)g.rows)[target * g.row_stride + c]), sum);
    dq[q * stride + c] = from_f32<T>(sum * by);
  }
}

// drows[row0 + j][c] = scale sum over the queries of G[q][j] q[q][c].  SPLIT: part[split][row][c] instead, of a split's queries.
// RESTS: also of what G's rounding left; else what that of the given rows' elements did.
template <typename T, bool SPLIT, bool RESTS>
__global__ __launch_bounds__(256, RESTS ? 2 : kGradWaves<T>) void grad_rows_kernel(GradArgs a, uint32_t row0, uint32_t rows, uint32_t ld, const T *__restrict__ G, const T *__restrict__ rests,
                                                        T *__restrict__ out, uint64_t stride, float *__restrict__ part, uint32_t splits) {
  const ScoreTable &g = a.g;
  __shared__ __attribute__((aligned(16))) char lds[kTileBytes<T, kAcross, kAcross>];
  const uint32_t c_tiles = (g.d + kTile - 1) / kTile, b8 = blockIdx.x / 8, split = SPLIT ? b8 % splits : 0, at = SPLIT ? b8 / splits : b8;
  const uint32_t ct = at % c_tiles, rt = at / c_tiles * 8 + blockIdx.x % 8;
  if (rt >= ld / kTile) return;
  const Lines<T> A = {G, ld, ld, g.nq}, B = {(const T *)g.q, g.q_stride, g.d, g.nq};
  uint32_t begin = 0, end = g.nq;
  if constexpr (SPLIT) {
    const uint32_t slices = (g.nq + Operand16<T>::kSlice - 1) / Operand16<T>::kSlice;
    begin = (uint32_t)((uint64_t)slices * split / splits) * Operand16<T>::kSlice;
    end = (uint32_t)((uint64_t)slices * (split + 1) / splits) * Operand16<T>::kSlice;
    if (end > g.nq) end = g.nq;
  }
  f32x16 acc[2][2];
  clear(acc);
  tile_product<T, kAcross, kAcross>(acc, A, rt * kTile, B, ct * kTile, begin, end, lds);
  if constexpr (RESTS) {
    const Lines<T> R = {rests, ld, ld, g.nq};
    tile_product<T, kAcross, kAcross>(acc, R, rt * kTile, B, ct * kTile, begin, end, lds);
  }
  const int wave = (int)threadIdx.x / kWave, lane = lane_id();
  if constexpr (sizeof(T) == 2) {
    if (!RESTS && a.targets) {
      // the queries whose given row is one of the tile's, in their order, 256 at a time
      uint32_t *list = (uint32_t *)lds;  // [256] queries, [256] rows of the tile, [4] counts
      const uint32_t tile0 = row0 + rt * kTile;
      for (uint32_t q0 = begin; q0 < end; q0 += 256) {
        const uint32_t q = q0 + threadIdx.x, at = (q < end ? a.targets[q] : ANN_PAD_ID) - tile0;
        const bool mine = at < kTile && tile0 + at < g.n && !(g.bias && g.bias[tile0 + at] == -INFINITY);
        const uint64_t of_wave = __ballot(mine);
        __syncthreads();  // the list has been read
        if (lane == 0) list[512 + wave] = __popcll(of_wave);
        __syncthreads();
        uint32_t place = __popcll(of_wave & ((1ull << lane) - 1)), count = 0;
        for (int w = 0; w < 4; ++w) {
          if (w < wave) place += list[512 + w];
          count += list[512 + w];
        }
        if (mine) list[place] = q, list[256 + place] = at;
        __syncthreads();
        for (uint32_t k = 0; k < count; ++k) {
          const uint32_t of = list[k], row = list[256 + k];
          if (row / 64 != (uint32_t)wave / 2) continue;
          const float rest = a.rest[of];
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const uint32_t c = ct * kTile + wave % 2 * 64 + j * 32 + lane % 32;
            const float v = c < g.d ? to_f32(((const T *)g.q)[of * g.q_stride + c]) : 0.0f;
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
              for (int r = 0; r < 16; ++r)
                if (row % 64 == (uint32_t)(i * 32 + block_row(r))) acc[i][j][r] = __builtin_fmaf(rest, v, acc[i][j][r]);
          }
        }
      }
    }
  }
  const float by = a.scaling ? g.scale * a.scaling[1] : g.scale;
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const uint32_t c = ct * kTile + wave % 2 * 64 + j * 32 + lane % 32;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const uint32_t row = rt * kTile + wave / 2 * 64 + i * 32 + block_row(r);
        if (row < rows && c < g.d) {
          if constexpr (SPLIT) {
            part[((uint64_t)split * rows + row) * g.d + c] = acc[i][j][r];
          } else {
            const bool left_out = g.bias && g.bias[row0 + row] == -INFINITY;  // (zero, whatever the queries hold)
            out[(uint64_t)(row0 + row) * stride + c] = from_f32<T>(left_out ? 0.0f : acc[i][j][r] * by);
          }
        }
      }
    }
}

// The splits' parts, in their order.
template <typename T>
__global__ __launch_bounds__(256) void grad_rows_sum_kernel(ScoreTable g, uint32_t row0, uint32_t rows, const float *__restrict__ part, uint32_t splits, T *__restrict__ out,
                                                            uint64_t stride, const float *__restrict__ scaling) {
  const uint64_t all = (uint64_t)rows * g.d, at = (uint64_t)blockIdx.x * 256 + threadIdx.x;
  if (at >= all) return;
  const float by = scaling ? g.scale * scaling[1] : g.scale;
  float sum = 0.0f;
  for (uint32_t s = 0; s < splits; ++s) sum += part[s * all + at];
  const uint64_t row = row0 + at / g.d;
  const bool left_out = g.bias && g.bias[row] == -INFINITY;
  out[row * stride + at % g.d] = from_f32<T>(left_out ? 0.0f : sum * by);
}

// Adds v with what the last addition lost: over many queries like terms lose with one sign (1.7e-4 of the sum of a million).
__device__ __forceinline__ void add_carried(float &sum, float &lost, float v) {
  v -= lost;
  const float next = sum + v;
  lost = (next - sum) - v;
  sum = next;
}

// drow_bias[row0 + j] = sum of the parts, in their order
__global__ __launch_bounds__(256) void grad_bias_kernel(const float *__restrict__ row_sums, uint32_t parts, uint32_t ld, uint32_t row0, uint32_t rows,
                                                        float *__restrict__ out) {
  const uint32_t j = blockIdx.x * 256 + threadIdx.x;
  if (j >= rows) return;
  float sum = 0.0f, lost = 0.0f;
  for (uint32_t p = 0; p < parts; ++p) add_carried(sum, lost, row_sums[(uint64_t)p * ld + j]);
  out[row0 + j] = sum;
}

// Short rows of 16 bits (KS slices of 16 columns): scores, G and its product in one kernel, G never leaving the registers.  A
// wavefront owns 32 lines of one side (OWN_ROWS: rows, otherwise queries), which stay in registers, and their gradient, 32 x 16 KS
// in accumulators; tiles of 64 lines of the other side pass by in LDS.  The scores' product puts the owned lines along
// the lanes and four by four of the passing ones into each lane's registers, and that is what the second product
// asks of its first operand if it takes the passing lines in that order (a sum has none); its second operand is the tile once more,
// transposed by the LDS.  Each side costs the scores anew: four products where storing G costs three, but G need not be
// written and read (twice two bytes for 256 operations).
// 4,096 x 100,000 x 128 bf16: 290 us for the queries' side, 329 for the rows' (730 and 640 TFLOP/s; 1,097 us with G stored).  Queries' side: vector
// instructions issue in 50 % of the cycles, LDS works in 39 (44 % of that conflicts), the matrix cores in 34: none of them bounds it alone,
// two wavefronts to a SIMD wait.  Rows' side: 26, 41 and 29, and 782 workgroups on 512 places.
constexpr int kPassing = 64, kOwned = 128;
constexpr uint32_t kShortTarget = 512;       // workgroups that own queries: two to a compute unit
constexpr uint64_t kShortStride = 1u << 24;  // row stride up to which offsets within a tile take 32 bits

template <typename T, int KS, bool OWN_ROWS, bool BIAS, bool ENTROPY>
__global__ __launch_bounds__(256, 2) void grad_short_kernel(GradArgs a, uint32_t splits, float *__restrict__ part, T *__restrict__ drows, uint64_t stride,
                                                            float *__restrict__ drow_bias) {
  typedef typename Operand16<T>::E E;
  constexpr int kSlots = 2 * KS, kLine = KS * 32 + 32, kUnits = kPassing * kSlots / 256;
  // (lines 32 bytes apart from a power of two: eight lines side by side hit all banks, and so do the four of a transposed read)
  __shared__ __attribute__((aligned(16))) char lds[2][kPassing * kLine];
  struct Line {  // of a passing line, in arrays so that four of them are one read
    float a[kPassing], b[kPassing], c[kPassing], d[kPassing];
    uint32_t target[kPassing];
  };
  __shared__ __attribute__((aligned(16))) Line info[2];
  const ScoreTable &g = a.g;
  const uint32_t owned = OWN_ROWS ? g.n : g.nq, passing = OWN_ROWS ? g.nq : g.n;
  const uint64_t own_stride = OWN_ROWS ? g.row_stride : g.q_stride, pass_stride = OWN_ROWS ? g.q_stride : g.row_stride;
  const T *own = (const T *)(OWN_ROWS ? g.rows : g.q), *pass = (const T *)(OWN_ROWS ? g.q : g.rows);
  const uint32_t own_tiles = (owned + kOwned - 1) / kOwned;
  // a die takes a run of rows through all queries
  const uint32_t b8 = blockIdx.x / 8, ot = OWN_ROWS ? blockIdx.x : b8 % own_tiles, split = OWN_ROWS ? 0 : b8 / own_tiles * 8 + blockIdx.x % 8;
  if (split >= splits) return;
  const uint32_t tiles = (passing + kPassing - 1) / kPassing;
  const uint32_t first = (uint32_t)((uint64_t)tiles * split / splits), last = (uint32_t)((uint64_t)tiles * (split + 1) / splits);
  const int wave = (int)threadIdx.x / kWave, lane = lane_id();
  const uint32_t own0 = ot * kOwned + wave * 32, mine = own0 + lane % 32;
  const float c = g.scale * kLog2e, scaling = a.scaling ? a.scaling[0] : 1.0f;
  E line[KS];
#pragma unroll
  for (int kk = 0; kk < KS; ++kk) {
    const uint32_t k = kk * 16 + lane / 32 * 8;
    Unit<T> u;
    load_unit(u, own + mine * own_stride + k, mine < owned ? (int64_t)g.d - k : 0);
    line[kk] = __builtin_bit_cast(E, u);
  }
  // Of a query: -lse, times log2 e without biases (-infinity: no row left, no probability); -g and -h, times the scaling; the entropy.
  const auto query = [&](uint32_t q, float &lse2, float &gl, float &gh, float &h, uint32_t &target) {
    const bool is = q < g.nq;
    target = is && a.targets ? a.targets[q] : ANN_PAD_ID;
    const float lse = is ? a.lse[q] : -INFINITY;
    lse2 = lse == -INFINITY ? -INFINITY : BIAS ? -lse : -lse * kLog2e;
    const bool none = lse == -INFINITY;
    gl = none || !a.g_logprob || target >= g.n ? 0.0f : -scaling * a.g_logprob[q];
    gh = ENTROPY && !none ? -scaling * a.g_entropy[q] : 0.0f;
    h = ENTROPY && !none ? a.entropy[q] : 0.0f;
  };
  float own_lse2 = 0.0f, own_gl = 0.0f, own_gh = 0.0f, own_h = 0.0f, own_bias = 0.0f;
  uint32_t own_target = ANN_PAD_ID;
  if constexpr (OWN_ROWS) {
    own_bias = mine < g.n ? (BIAS ? g.bias[mine] : 0.0f) : -INFINITY;
  } else {
    query(mine, own_lse2, own_gl, own_gh, own_h, own_target);
  }
  Unit<T> u[kUnits];
  float unit_bias[kUnits];
  uint32_t from[kUnits], to[kUnits];
#pragma unroll
  for (int i = 0; i < kUnits; ++i) {
    const uint32_t at = threadIdx.x + 256 * i, l = at / kSlots, slot = at % kSlots;
    from[i] = (l * (uint32_t)pass_stride + slot * 8) * sizeof(T);
    to[i] = l * kLine + slot * 16;
    unit_bias[i] = 0.0f;
  }
  const auto fetch = [&](uint32_t tile) {
    const T *base = pass + (uint64_t)tile * kPassing * pass_stride;
    if (KS * 16 == g.d && (tile + 1) * kPassing <= passing && pass_stride <= kShortStride) {
#pragma unroll
      for (int i = 0; i < kUnits; ++i) load_unit(u[i], (const T *)((const char *)base + from[i]));
    } else {
#pragma unroll
      for (int i = 0; i < kUnits; ++i) {
        const uint32_t at = threadIdx.x + 256 * i, l = at / kSlots, k = at % kSlots * 8;
        load_unit(u[i], base + l * pass_stride + k, tile * kPassing + l < passing ? (int64_t)g.d - k : 0);
      }
    }
    if (BIAS && !OWN_ROWS) {
#pragma unroll
      for (int i = 0; i < kUnits; ++i) {
        const uint32_t l = tile * kPassing + (threadIdx.x + 256 * i) / kSlots;
        unit_bias[i] = l < passing ? g.bias[l] : -INFINITY;
      }
    }
  };
  f32x16 acc[KS / 2];
#pragma unroll
  for (int b = 0; b < KS / 2; ++b)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[b][r] = 0.0f;
  float sum = 0.0f, sum_lost = 0.0f;  // of the owned row's elements of G
  if (first < last) fetch(first);
  for (uint32_t tile = first; tile < last; ++tile) {
    char *at = lds[tile & 1];
    Line &of = info[tile & 1];
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
      uint4 v = unit_part(u[i], 0);
      if (BIAS && !OWN_ROWS && unit_bias[i] == -INFINITY) v = make_uint4(0, 0, 0, 0);  // (rows left out may hold anything)
      *(uint4 *)(at + to[i]) = v;
    }
    const bool whole = tile * kPassing + kPassing <= passing;
    if (threadIdx.x < kPassing) {
      const uint32_t l = tile * kPassing + threadIdx.x;
      if constexpr (OWN_ROWS)
        query(l, of.a[threadIdx.x], of.b[threadIdx.x], of.c[threadIdx.x], of.d[threadIdx.x], of.target[threadIdx.x]);
      else if (BIAS || !whole)
        of.a[threadIdx.x] = l < passing ? (BIAS ? g.bias[l] : 0.0f) : -INFINITY;
    }
    __syncthreads();  // (one per tile: whoever writes this half again has met the others at the next tile's)
    if (tile + 1 < last) fetch(tile + 1);
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      f32x16 s;
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = 0.0f;
      const char *x = at + (half * 32 + lane % 32) * kLine + lane / 32 * 16;
#pragma unroll
      for (int kk = 0; kk < KS; ++kk) s = matrix_step(*(const E *)(x + kk * 32), line[kk], s);
      // G, times the scaling
      const uint32_t line0 = tile * kPassing + half * 32;
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        const int l = half * 32 + block_row(r);
        float lse2[4], gl[4], gh[4], h[4], bias[4];
        if constexpr (OWN_ROWS) {
          *(float4 *)lse2 = *(const float4 *)(of.a + l), *(float4 *)gl = *(const float4 *)(of.b + l);
          if (ENTROPY) *(float4 *)gh = *(const float4 *)(of.c + l), *(float4 *)h = *(const float4 *)(of.d + l);
        } else if (BIAS || !whole) {
          *(float4 *)bias = *(const float4 *)(of.a + l);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float b = OWN_ROWS ? own_bias : BIAS || !whole ? bias[e] : 0.0f;
          // log2 p (biases may be as low as they get: in natural units nothing overflows)
          float y = OWN_ROWS ? lse2[e] : own_lse2;
          y = BIAS ? (__builtin_fmaf(s[r + e], g.scale, b) + y) * kLog2e : __builtin_fmaf(s[r + e], c, y);
          const float p = __builtin_amdgcn_exp2f(y);
          float slope = OWN_ROWS ? gl[e] : own_gl;
          if (ENTROPY) slope = __builtin_fmaf(OWN_ROWS ? gh[e] : own_gh, __builtin_fmaf(y, kLn2, OWN_ROWS ? h[e] : own_h), slope);
          float v = p * slope;
          // (no probability: 0, also where log p is -infinity and the slope with it; rows left out likewise, whatever they hold)
          if (ENTROPY && !(p != 0.0f)) v = 0.0f;
          if ((BIAS || (!OWN_ROWS && !whole)) && b == -INFINITY) v = 0.0f;
          s[r + e] = v;
        }
      }
      // the given rows' elements: few blocks have one
      const uint32_t target = OWN_ROWS ? of.target[half * 32 + lane % 32] : own_target;
      const uint32_t hit = target - (OWN_ROWS ? own0 : line0);
      const bool hits = __any(hit < 32 && target < g.n);
      if (hits) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int l = block_row(r);
          if constexpr (OWN_ROWS) {
            if (of.target[half * 32 + l] == mine && mine < g.n && own_bias != -INFINITY) s[r] -= of.b[half * 32 + l];
          } else {
            if (hit == (uint32_t)l && target < g.n && !(BIAS && of.a[half * 32 + l] == -INFINITY)) s[r] -= own_gl;
          }
        }
      }
      if (OWN_ROWS && drow_bias) {
        float some = 0.0f;
#pragma unroll
        for (int r = 0; r < 16; ++r) some += s[r];
        add_carried(sum, sum_lost, some);
      }
      E G[2];
#pragma unroll
      for (int r = 0; r < 16; ++r) G[r / 8][r % 8] = from_f32<T>(s[r]);
      if (!OWN_ROWS && hits) {
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (hit == (uint32_t)block_row(r) && target < g.n) a.rest[mine] = s[r] - to_f32((T)G[r / 8][r % 8]);
      }
      // lines 16 t + 4 (lane / 32) + 0 .. 3 and 8 further are the lane's eight k of step t
      const auto multiply = [&](const E(&by)[2]) {
#pragma unroll
        for (int b = 0; b < KS / 2; ++b)
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            union {
              s16x4 part[2];
              E e;
            } f;
#pragma unroll
            for (int p = 0; p < 2; ++p) {
              const int l = half * 32 + t * 16 + p * 8 + lane / 32 * 4 + lane % 16 / 4, column = b * 32 + lane / 16 % 2 * 16 + lane % 4 * 4;
              f.part[p] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(at + l * kLine + column * 2));
            }
            acc[b] = matrix_step(by[t], f.e, acc[b]);
          }
      };
      multiply(G);
      if (OWN_ROWS && (hits || g.nq <= kFewQueries)) {  // what the rounding left, in 16 bits more
#pragma unroll
        for (int r = 0; r < 16; ++r) G[r / 8][r % 8] = from_f32<T>(s[r] - to_f32((T)G[r / 8][r % 8]));
        multiply(G);
      }
    }
  }
  if (OWN_ROWS && drow_bias) {
    const LanePair p = lane_pair<false>(__float_as_uint(sum));
    sum = __uint_as_float(p.low) + __uint_as_float(p.high);
    if (lane < 32 && mine < g.n) drow_bias[mine] = sum / scaling;
  }
  if (OWN_ROWS && !drows) return;
  const float by = a.scaling ? g.scale * a.scaling[1] : g.scale;
#pragma unroll
  for (int b = 0; b < KS / 2; ++b) {
    const uint32_t column = b * 32 + lane % 32;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const uint32_t l = own0 + block_row(r);
      if (l >= owned || column >= g.d) continue;
      if constexpr (OWN_ROWS) {
        const bool left_out = BIAS && g.bias[l] == -INFINITY;  // (zero, whatever the queries hold)
        drows[l * stride + column] = from_f32<T>(left_out ? 0.0f : acc[b][r] * by);
      } else {
        part[((uint64_t)split * g.nq + l) * g.d + column] = acc[b][r];
      }
    }
  }
}

// ---------------------------------------------------------------------------
struct BackwardPlan {
  uint32_t q_tiles = 0, chunk = 0, splits = 0;  // chunk: rows at a time, a multiple of kTile
  uint32_t row_splits = 1;                      // of the queries, in the rows' product
  int slices = 0;                               // of 16 columns, if G stays in registers
  bool wide = false;                            // the queries' product: tiles of 256 of them
  uint64_t g_at = 0, rests_at = 0, part_at = 0, row_part_at = 0, sums_at = 0, scaling_at = 0, rest_at = 0;
  Parts parts;
};

static BackwardPlan backward_plan(uint32_t nq, uint64_t n, uint32_t d, uint32_t type) {
  BackwardPlan p;
  if (nq == 0 || n == 0) return p;
  p.q_tiles = (nq + kTile - 1) / kTile;
  if (type != ANN_F32 && d <= 128) {
    p.slices = d <= 64 ? 4 : d <= 96 ? 6 : 8;
    const uint32_t tiles = (uint32_t)((n + kPassing - 1) / kPassing), want = ((kShortTarget + p.q_tiles - 1) / p.q_tiles + 7) / 8 * 8;
    p.splits = want < tiles ? want : tiles;
    p.part_at = p.parts.take((uint64_t)p.splits * nq * d * sizeof(float));
    p.scaling_at = p.parts.take(2 * sizeof(float));
    p.rest_at = p.parts.take(nq * sizeof(float));
    return p;
  }
  const uint64_t row_bytes = (uint64_t)nq * type_bytes(type), all = (n + kTile - 1) / kTile * kTile;
  uint64_t chunk = kChunkBytes / row_bytes / kTile * kTile;
  if (chunk < kTile) chunk = kTile;
  if (chunk > all) chunk = all;
  // chunks of like sizes
  const uint64_t chunks = (all + chunk - 1) / chunk;
  p.chunk = (uint32_t)((all / kTile + chunks - 1) / chunks * kTile);
  const uint32_t c_tiles = (d + kTile - 1) / kTile, most = (p.chunk + 255) / 256;
  p.wide = type != ANN_F32 && d % 8 == 0 && nq > kTile && (uint64_t)p.q_tiles * (p.chunk / kTile) >= 2 * kWideSlots;
  if (p.wide) {
    // Rounds of workgroups times slices of each (1.3 us: 512 workgroups at 850 TFLOP/s), and the parts written and read at 4 TB/s.
    const uint32_t tiles = (nq + kWideM - 1) / kWideM * c_tiles, slices = p.chunk / kWideSlice;
    double least = INFINITY;
    for (uint32_t s = 1; s <= 64 && s <= most; ++s) {
      const double cost = 1.3 * (((uint64_t)tiles * s + kWideSlots - 1) / kWideSlots) * ((slices + s - 1) / s) + 2e-6 * s * nq * d;
      if (cost < least) least = cost, p.splits = s;
    }
  } else {
    const uint32_t tiles = p.q_tiles * c_tiles;
    p.splits = ((kGradTarget + tiles - 1) / tiles + 7) / 8 * 8;
    if (p.splits > most) p.splits = most;
  }
  p.g_at = p.parts.take(p.chunk * row_bytes);
  if (type != ANN_F32 && nq <= kFewQueries) p.rests_at = p.parts.take(p.chunk * row_bytes);
  p.part_at = p.parts.take((uint64_t)p.splits * nq * d * sizeof(float));
  // (one chunk whose tiles leave compute units with one workgroup or none: runs of queries, of 64 at least)
  const uint32_t row_tiles = p.chunk / kTile * c_tiles;
  if (chunks == 1 && row_tiles < 512) {
    p.row_splits = (kGradTarget + row_tiles - 1) / row_tiles;
    if (p.row_splits > (nq + 63) / 64) p.row_splits = (nq + 63) / 64;
    if (p.row_splits > 8) p.row_splits = 8;
  }
  if (p.row_splits > 1) p.row_part_at = p.parts.take((uint64_t)p.row_splits * n * d * sizeof(float));
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
  T *G = (T *)(ws + p.g_at), *rests = sizeof(T) == 2 && g.nq && g.nq <= kFewQueries && o.drows ? (T *)(ws + p.rests_at) : nullptr;
  float *part = (float *)(ws + p.part_at), *sums = (float *)(ws + p.sums_at);
  a.rest = (float *)(ws + p.rest_at);
  if (sizeof(T) == 2 && std::is_same<T, f16_t>::value && g.nq && g.n) {
    float *scaling = (float *)(ws + p.scaling_at);
    grad_scaling_kernel<<<1, 1024, 0, st>>>(a, scaling);
    ANN_HIP(hipGetLastError());
    a.scaling = scaling;
  }
  if (p.slices) {
    const auto run = [&](auto slices, auto bias, auto entropy) {
      if constexpr (sizeof(T) == 2) {
        constexpr int KS = decltype(slices)::value;
        constexpr bool BIAS = decltype(bias)::value, ENTROPY = decltype(entropy)::value;
        if (o.dq)
          grad_short_kernel<T, KS, false, BIAS, ENTROPY><<<p.q_tiles * ((p.splits + 7) / 8 * 8), 256, 0, st>>>(a, p.splits, part, nullptr, 0, nullptr);
        if (o.drows || o.drow_bias)
          grad_short_kernel<T, KS, true, BIAS, ENTROPY><<<(g.n + kOwned - 1) / kOwned, 256, 0, st>>>(a, 1, nullptr, (T *)o.drows, o.drows_stride, o.drow_bias);
      }
    };
    const auto run_entropy = [&](auto slices, auto bias) {
      if (a.g_entropy)
        run(slices, bias, std::true_type());
      else
        run(slices, bias, std::false_type());
    };
    const auto run_bias = [&](auto slices) {
      if (g.bias)
        run_entropy(slices, std::true_type());
      else
        run_entropy(slices, std::false_type());
    };
    if (p.slices == 4)
      run_bias(std::integral_constant<int, 4>());
    else if (p.slices == 6)
      run_bias(std::integral_constant<int, 6>());
    else
      run_bias(std::integral_constant<int, 8>());
    ANN_HIP(hipGetLastError());
    if (o.dq) {
      // (256 splits of 256 queries: 15.5 us by two wavefronts to a query)
      if (p.splits >= 64)
        grad_queries_sum_kernel<T, 128, 8, 1024><<<g.nq, 1024, 0, st>>>(a, part, p.splits, (T *)o.dq, o.dq_stride);
      else
        grad_queries_sum_kernel<T, 128, 1, 256><<<(g.nq + 1) / 2, 256, 0, st>>>(a, part, p.splits, (T *)o.dq, o.dq_stride);
      ANN_HIP(hipGetLastError());
    }
    return ANN_OK;
  }
  // (no queries: one chunk of all rows, of which no product takes anything)
  const uint32_t chunk = p.chunk ? p.chunk : (g.n + kTile - 1) / kTile * kTile;
  for (uint32_t row0 = 0; row0 < g.n; row0 += chunk) {
    const uint32_t rows = g.n - row0 < chunk ? g.n - row0 : chunk, ld = (rows + kTile - 1) / kTile * kTile;
    if (g.nq) {
      const uint32_t grid = p.q_tiles * ((ld / kTile + 7) / 8 * 8);
      const auto run = [&](auto bias, auto entropy, auto row_sums) {
        grad_scores_kernel<T, decltype(bias)::value, decltype(entropy)::value, decltype(row_sums)::value><<<grid, 256, 0, st>>>(a, row0, p.q_tiles, ld, G, rests, sums);
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
        const auto product = [&](auto blocks) {
          constexpr int MB = decltype(blocks)::value;
          const uint32_t tiles = c_tiles * ((g.nq + MB * 64 - 1) / (MB * 64)) * p.splits;
          grad_queries_kernel<T, MB><<<(tiles + 7) / 8 * 8, 256, 0, st>>>(g, row0, rows, ld, G, p.splits, part, row0 != 0);
        };
        // (biases: rows left out may hold anything, which the wide product does not look for)
        if (p.wide && !g.bias && wide_operand(g.rows, g.row_stride)) {
          if constexpr (sizeof(T) == 2) product(std::integral_constant<int, 4>());
        } else {
          product(std::integral_constant<int, 2>());
        }
        ANN_HIP(hipGetLastError());
      }
    }
    if (o.drows) {
      const uint32_t grid = c_tiles * ((ld / kTile + 7) / 8 * 8) * p.row_splits;
      float *row_part = (float *)(ws + p.row_part_at);
      const auto product = [&](auto split, auto with_rests) {
        grad_rows_kernel<T, decltype(split)::value, decltype(with_rests)::value>
            <<<grid, 256, 0, st>>>(a, row0, rows, ld, G, rests, (T *)o.drows, o.drows_stride, row_part, p.row_splits);
      };
      const auto with_split = [&](auto split) {
        if (sizeof(T) == 2 && rests)
          product(split, std::integral_constant<bool, sizeof(T) == 2>());
        else
          product(split, std::false_type());
      };
      if (p.row_splits > 1) {
        with_split(std::true_type());
        ANN_HIP(hipGetLastError());
        grad_rows_sum_kernel<T><<<(uint32_t)(((uint64_t)rows * g.d + 255) / 256), 256, 0, st>>>(g, row0, rows, row_part, p.row_splits, (T *)o.drows, o.drows_stride, a.scaling);
      } else {
        with_split(std::false_type());
      }
      ANN_HIP(hipGetLastError());
    }
    if (o.drow_bias) {
      grad_bias_kernel<<<(rows + 255) / 256, 256, 0, st>>>(sums, p.q_tiles * 2, ld, row0, rows, o.drow_bias);
      ANN_HIP(hipGetLastError());
    }
  }
  if (o.dq && g.nq) {
    grad_queries_sum_kernel<T, 256, 1, 256><<<g.nq, 256, 0, st>>>(a, part, g.n ? p.splits : 0, (T *)o.dq, o.dq_stride);
    ANN_HIP(hipGetLastError());
  }
  return ANN_OK;
}

}  // namespace ann

using namespace ann;

extern "C" uint64_t ann_row_logprobs_backward_workspace(uint32_t nq, uint64_t n, uint32_t d, uint32_t type) {
  if (n > kMaxRows || nq >= kMaxQueries || d == 0 || type > ANN_BF16) return 0;
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
