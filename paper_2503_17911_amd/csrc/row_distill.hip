// Distillation: how far the softmax of all rows' scores is from a teacher's k likeliest rows and their probabilities, and its gradients.
//
//   t_ie = exp(given_ie),  loss_i = sum_e t_ie (given_ie - log p_i[id_ie]),  T_i = sum_e t_ie
//   G[i][j] = g_i (T_i p_ij - sum of t_ie over the entries e with id_ie = j),   dq = scale G X,  dX = scale G^T Q,  dbias = sum_i G_i
//
// (Short lists have kernels of their own, below.)
// Forward: the log of the softmax' sum over all rows is that of the rows' log probabilities; the given rows' scores are formed again (fp64 sums).
// Backward: G has a part at all rows and one at k rows of each query.  The first is what the rows' log probabilities have, with the weight
// -g_i T_i: its kernels, with G of 16-bit rows in two parts of 16 bits (2^-18 of an element is left in bf16, 2^-24 in f16): where the student is near the
// teacher, or its likely rows are alike, the products are small differences, and the rounding of g T p to 16 bits would be seen in them.  The second is
// added in fp32 to the products' results before these are rounded.  For dq that is a sum of k rows to a query.  For the rows the entries are put in the
// order of their ids and summed by runs, so that a row that many teachers name costs no more than others.
// Measured: gradients of 4,096 x 100,000 x 128 bf16 with k = 32: 619 us, of which the first part takes 570 (bound as its kernels are; 714 the call where every
// block has a likely row), the order of the entries 27, their runs and join 25, the entries and the queries' sums 13.  Forward: 8 x 1M x 128 55 us, 5 of them
// for the given rows; 4,096 x 100,000 x 128 221 us in bf16, 217 in f16, 1,011 in fp32, whose scores take the smaller products of their parts apart (the rows'
// log probabilities, which do not, 690): losses are differences of log probabilities, off by 2.6e-8 so, and small where the student is near its teacher.
#include "row_logprobs.hpp"
#include "row_runs.hpp"

#include <math.h>

namespace ann {

// Of an entry: its log probability under the student (0: no row is given, -infinity: the row is left out), and of a query: its loss.  16 lanes to an entry.
template <typename T>
__global__ __launch_bounds__(256) void distill_loss_kernel(ScoreTable g, uint32_t k, const uint32_t *__restrict__ ids, const float *__restrict__ given,
                                                           const double *__restrict__ lse, float *__restrict__ loss, float *__restrict__ logprobs) {
  constexpr int VEC = 16 / (int)sizeof(T);
  __shared__ double terms[ANN_MAX_ALTERNATIVES];
  const uint32_t q = blockIdx.x, lane = threadIdx.x % 16;
  const double l = lse[q];  // (rounded to fp32 it would move every log probability by up to half a step of lse)
  for (uint32_t e = threadIdx.x / 16; e < k; e += 16) {
    const uint32_t id = ids[(uint64_t)q * k + e];
    const float bias = id < g.n && g.bias ? g.bias[id] : 0.0f;
    double sum = 0.0;
    if (id < g.n && bias != -INFINITY) {
      const T *x = (const T *)g.rows + id * g.row_stride, *y = (const T *)g.q + q * g.q_stride;
      for (uint32_t c = lane * VEC; c < g.d; c += 16 * VEC) {
        RowPiece<T, VEC, kShifted> a, b;
        a.load(x, c, g.d), b.load(y, c, g.d);
#pragma unroll
        for (int i = 0; i < VEC; ++i) sum += (double)a.get(i) * (double)b.get(i);
      }
    }
    sum = group_sum_f64<16>(sum);
    if (lane != 0) continue;
    double logp = 0.0;
    if (id < g.n) logp = bias == -INFINITY ? -INFINITY : sum * (double)g.scale + (double)bias - l;
    logp = logp > 0.0 ? 0.0 : logp;  // (what lse is off, where the row has all probability)
    logprobs[(uint64_t)q * k + e] = (float)logp;
    const double t = id < g.n ? (double)given[(uint64_t)q * k + e] : -INFINITY, weight = exp(t);
    terms[e] = weight == 0.0 ? 0.0 : weight * (t - logp);  // (without a weight nothing counts, also where logp is -infinity)
  }
  __syncthreads();
  if (threadIdx.x != 0) return;
  double sum = 0.0;
  for (uint32_t e = 0; e < k; ++e) sum += terms[e];
  loss[q] = (float)sum;
}

// Forward of short lists, such as a batch's own rows: all scores in fp64, from fp64 matrix instructions (a product of two fp32 numbers is whole in 64 bits),
// kept in the workspace; then a wavefront to a query sums them and finds the given rows' among them.  So what a student near its teacher loses is not the
// difference of two roundings, and the given rows are not read again.  A workgroup makes 16 x 16 scores, each wavefront along a quarter of the columns; it is
// bound by the matrix instructions (16 x 16 x 4 in 64 cycles) once the card is full.  Two blocks of rows to a wavefront won 1 to 5% for 16 bits, 15% for the largest in
// fp32, and lost as much with few queries: one.
// Measured, us, here against the kernels for long lists (k = 20, bf16 / fp32): 8 x 256 x 960 12 / 12 against 32 / 58; 300 x 256 x 960 13 / 14 against 36 / 87;
// 3,000 x 128 x 768 22 / 26 against 47 / 91; 3,000 x 256 x 960 40 / 49 against 56 / 113; 30,000 x 256 x 960 321 / 415 against 350 / 570 (k = 1: 320 / 415 against
// 227 / 414, k = 64: 321 / 415 against 839 / 1,004).  Longer lists gain while the work is small: 300 x 1,024 x 960 27 against 36, 1,500 x 512 x 960 42 against 41,
// but 300 x 2,048 x 960 47 against 36, 4,096 x 512 x 960 93 against 68, 4,096 x 1,024 x 128 48 against 28 (bf16).
constexpr uint64_t kShortRows = 256, kShortScores = 1ull << 23;                                 // at most 64 MiB of workspace
constexpr uint64_t kMiddleRows = 1024, kMiddleScores = 1ull << 20, kMiddleWork = 3ull << 28;  // (products)
static bool short_list(uint64_t nq, uint64_t n, uint32_t d) {
  if (n == 0 || n > kMiddleRows) return false;
  return n <= kShortRows ? nq * n <= kShortScores : nq * n <= kMiddleScores && nq * n * d <= kMiddleWork;
}

template <typename T, RowEnd END>
__global__ __launch_bounds__(256) void distill_short_kernel(ScoreTable g, uint32_t row_tiles, double *__restrict__ scores) {
  typedef double f64x4 __attribute__((ext_vector_type(4)));
  constexpr uint32_t kStep = 32;  // columns: 8 to a lane, of the four lanes that hold a row
  __shared__ double parts[4][256];
  const uint32_t wave = threadIdx.x / kWave, lane = threadIdx.x % kWave, q0 = blockIdx.x / row_tiles * 16, r0 = blockIdx.x % row_tiles * 16;
  const uint32_t query = q0 + lane % 16 < g.nq ? q0 + lane % 16 : g.nq - 1, row = r0 + lane % 16 < g.n ? r0 + lane % 16 : g.n - 1;
  const T *y = (const T *)g.q + query * g.q_stride, *x = (const T *)g.rows + row * g.row_stride;
  f64x4 sum = {0.0, 0.0, 0.0, 0.0};
  RowPiece<T, 8, END> a, b;
  uint32_t c = wave * kStep;
  if (c < g.d) a.load(y, c + lane / 16 * 8, g.d), b.load(x, c + lane / 16 * 8, g.d);
  while (c < g.d) {
    const RowPiece<T, 8, END> of_q = a, of_x = b;
    c += 4 * kStep;
    if (c < g.d) a.load(y, c + lane / 16 * 8, g.d), b.load(x, c + lane / 16 * 8, g.d);
#pragma unroll
    for (int e = 0; e < 8; ++e) sum = __builtin_amdgcn_mfma_f64_16x16x4f64((double)of_q.get(e), (double)of_x.get(e), sum, 0, 0, 0);
  }
  // (register e of a lane: query lane / 16 + 4 e, row lane % 16)
#pragma unroll
  for (int e = 0; e < 4; ++e) parts[wave][e * kWave + lane] = sum[e];
  __syncthreads();
  const uint32_t t = threadIdx.x, i = q0 + t / 16, j = r0 + t % 16;
  if (i >= g.nq || j >= g.n) return;
  const float bias = g.bias ? g.bias[j] : 0.0f;
  const double dot = (parts[0][t] + parts[1][t]) + (parts[2][t] + parts[3][t]);
  scores[(uint64_t)i * g.n + j] = bias == -INFINITY ? -INFINITY : dot * (double)g.scale + (double)bias;
}

template <typename T>
static void launch_short(const ScoreTable &g, double *scores, hipStream_t st) {
  const uint32_t row_tiles = (g.n + 15) / 16, tiles = (g.nq + 15) / 16 * row_tiles;
  if (g.d % 8 == 0)
    distill_short_kernel<T, kWholePieces><<<tiles, 256, 0, st>>>(g, row_tiles, scores);
  else
    distill_short_kernel<T, kShifted><<<tiles, 256, 0, st>>>(g, row_tiles, scores);
}

__global__ __launch_bounds__(256) void distill_short_loss_kernel(uint32_t nq, uint32_t n, const double *__restrict__ scores, uint32_t k, const uint32_t *__restrict__ ids,
                                                                 const float *__restrict__ given, float *__restrict__ loss, float *__restrict__ lse_out,
                                                                 float *__restrict__ logprobs) {
  constexpr float kLargest = 3.402823466e38f;
  const uint32_t q = blockIdx.x * 4 + threadIdx.x / kWave, lane = threadIdx.x % kWave;
  if (q >= nq) return;
  const double *s = scores + (uint64_t)q * n;
  const uint64_t at = (uint64_t)q * k + lane;
  const uint32_t id = lane < k ? ids[at] : ANN_PAD_ID;
  const double t = id < n ? (double)given[at] : -INFINITY, weight = exp(t);
  const double own = id < n ? s[id] : 0.0;
  float top = -INFINITY;
  for (uint32_t j = lane; j < n; j += kWave) top = fmaxf(top, (float)s[j]);
  top = fmaxf(-kLargest, fminf(lanes_max(top, kWave), kLargest));
  double sum = 0.0;
  for (uint32_t j = lane; j < n; j += kWave) sum += exp(s[j] - (double)top);
  sum = group_sum_f64<kWave>(sum);
  const double lse = sum == 0.0 ? -INFINITY : (double)top + log(sum);
  const double above = id >= n ? 0.0 : own == -INFINITY ? -INFINITY : own - lse, logp = above > 0.0 ? 0.0 : above;  // (what lse is off)
  const double all = group_sum_f64<kWave>(weight == 0.0 ? 0.0 : weight * (t - logp));  // (without a weight nothing counts, also where logp is -infinity)
  if (lane < k) logprobs[at] = (float)logp;
  if (lane == 0) loss[q] = (float)all, lse_out[q] = (float)lse;
}

// Backward of short lists: the scores in fp64 as above, G from them in their place (both parts together, so nothing is left to add), and both products by the fp64 matrix
// instructions: G X and G^T Q in one launch.  A workgroup makes 16 rows of 64 columns, each of its eight wavefronts along every eighth block of four of the sum; it reads
// a block of 16 ahead (without: 63 us in the place of 43 for 3,000 x 64 x 96, where eight workgroups make all of G^T Q; with more queries than 4,096 that is too few).
// Measured, us, here against the kernels for long lists (k = 20, bf16 / fp32): 8 x 256 x 960 18 / 19 against 66 / 115; 300 x 256 x 960 30 / 31 against 91 / 146;
// 3,000 x 128 x 768 71 / 75 against 124 / 187; 3,000 x 64 x 96 52 / 54 against 64 / 96; 4,096 x 256 x 960 162 / 168 against 164 / 261 (k = 1, bf16: 155 against 135;
// k = 64: 159 against 197); 300 x 1,024 x 960 71 / 75 against 100 / 153.
static bool short_gradient(uint64_t nq, uint64_t n, uint32_t d) { return nq && nq <= 4096 && short_list(nq, n, d); }

__global__ __launch_bounds__(256) void distill_short_weights_kernel(uint32_t nq, uint32_t n, double *__restrict__ scores, uint32_t k, const uint32_t *__restrict__ ids,
                                                                    const float *__restrict__ given, const float *__restrict__ lse, const float *__restrict__ g_loss) {
  // a wavefront's own: its query's entries, and a bit to each row that one of them names
  __shared__ uint32_t all_ids[4][kWave], all_named[4][kMiddleRows / 32];
  __shared__ double all_weights[4][kWave];
  const uint32_t wave = threadIdx.x / kWave, lane = threadIdx.x % kWave, q = blockIdx.x * 4 + wave < nq ? blockIdx.x * 4 + wave : nq - 1;
  const uint64_t at = (uint64_t)q * k + lane;
  const uint32_t id = lane < k ? ids[at] : ANN_PAD_ID;
  const double t = id < n ? exp((double)given[at]) : 0.0, whole = group_sum_f64<kWave>(t);
  double *s = scores + (uint64_t)q * n;
  const double own = id < n ? s[id] : 0.0;
  all_ids[wave][lane] = id, all_weights[wave][lane] = t;
  for (uint32_t w = lane; w < kMiddleRows / 32; w += kWave) all_named[wave][w] = 0;
  __syncthreads();
  if (id < n) atomicOr(&all_named[wave][id / 32], 1u << id % 32);
  // the weights of a row that is named more than once, by the first that names it
  bool first = id < n;
  double sum = 0.0;
  for (uint32_t e = 0; e < k; ++e) {
    const bool same = all_ids[wave][e] == id;
    if (same && e < lane) first = false;
    sum += same ? all_weights[wave][e] : 0.0;
  }
  __syncthreads();
  if (blockIdx.x * 4 + wave >= nq) return;
  const double l = (double)lse[q], g = (double)g_loss[q];
  const bool none = lse[q] == -INFINITY;
  // (-infinity: the row is left out)
  if (first) s[id] = none || own == -INFINITY ? 0.0 : g * (whole * exp(own - l) - sum);
  for (uint32_t j = lane; j < n; j += kWave)
    if (!(all_named[wave][j / 32] >> j % 32 & 1)) s[j] = none || s[j] == -INFINITY ? 0.0 : g * (whole * exp(s[j] - l));
}

template <typename T, RowEnd END>
__global__ __launch_bounds__(512) void distill_short_grad_kernel(ScoreTable g, const double *__restrict__ weights, const float *__restrict__ lse, GradOut o, uint32_t row_tiles,
                                                                 uint32_t row_columns, uint32_t q_columns) {
  typedef double f64x4 __attribute__((ext_vector_type(4)));
  constexpr int kWaves = 8, kAhead = 4;
  __shared__ double parts[kWaves][4][256];
  __shared__ double bias_parts[kWaves][kWave];
  const uint32_t wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
  const bool by_row = blockIdx.x < row_tiles;  // (their sums are longer: first)
  const uint32_t tile = by_row ? blockIdx.x : blockIdx.x - row_tiles, columns = by_row ? row_columns : q_columns;
  const uint32_t m0 = tile / columns * 16, c0 = tile % columns * 64, count = by_row ? g.n : g.nq, along = by_row ? g.nq : g.n;
  const uint32_t i = m0 + lane % 16 < count ? m0 + lane % 16 : count - 1, c = c0 + lane % 16 * 4;
  const T *from = (const T *)(by_row ? g.q : g.rows);
  const uint64_t stride = by_row ? g.q_stride : g.row_stride;
  f64x4 sum[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) sum[e] = {0.0, 0.0, 0.0, 0.0};
  double of_bias = 0.0;
  const float *marks = by_row ? lse : g.bias;  // -infinity: what the row holds is nothing (it is left out, the query has no row left)
  double next_a[kAhead];
  RowPiece<T, 4, END> next_b[kAhead];
  float next_mark[kAhead];
  const auto load = [&](uint32_t start) {
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const uint32_t at = start + u * kWaves * 4 + lane / 16, j = at < along ? at : along - 1;
      next_a[u] = weights[by_row ? (uint64_t)j * g.n + i : (uint64_t)i * g.n + j];
      next_b[u].load(from + j * stride, c, g.d);
      next_mark[u] = marks ? marks[j] : 0.0f;
    }
  };
  uint32_t start = wave * 4;
  if (start < along) load(start);
  while (start < along) {
    double a[kAhead];
    RowPiece<T, 4, END> b[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const bool there = start + u * kWaves * 4 + lane / 16 < along;
      a[u] = there ? next_a[u] : 0.0, b[u] = next_b[u];
      if (!there || next_mark[u] == -INFINITY) b[u].clear();
    }
    const uint32_t now = start;
    start += kWaves * 4 * kAhead;
    if (start < along) load(start);
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if (now + u * kWaves * 4 >= along) break;
      of_bias += a[u];
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[e] = __builtin_amdgcn_mfma_f64_16x16x4f64(a[u], (double)b[u].get(e), sum[e], 0, 0, 0);
    }
  }
#pragma unroll
  for (int e = 0; e < 4; ++e)
#pragma unroll
    for (int r = 0; r < 4; ++r) parts[wave][e][r * kWave + lane] = sum[e][r];
  bias_parts[wave][lane] = of_bias;
  __syncthreads();
  const uint32_t t = threadIdx.x, to = m0 + t / 16 % 16;
  if (t >= 256 || to >= count) return;
  // no row left for the query, the row left out: zero, whatever the others hold
  const bool nothing = by_row ? g.bias && g.bias[to] == -INFINITY : lse[to] == -INFINITY;
  if (by_row && o.drow_bias && c0 == 0 && t % 16 == 0) {
    double v = 0.0;
    for (int w = 0; w < kWaves; ++w)
      for (int h = 0; h < 4; ++h) v += bias_parts[w][h * 16 + t / 16];
    o.drow_bias[to] = nothing ? 0.0f : (float)v;
  }
  T *out = (T *)(by_row ? o.drows : o.dq);
  if (!out) return;
  float v[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    double whole = 0.0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) whole += parts[w][e][t];
    v[e] = nothing ? 0.0f : (float)(whole * (double)g.scale);
  }
  RowPiece<T, 4> piece;
  piece.set(v);
  piece.store(out + to * (by_row ? o.drows_stride : o.dq_stride), c0 + t % 16 * 4, g.d);
}

template <typename T>
static ann_status short_backward(const GradArgs &a, const GradOut &o, uint32_t k, const uint32_t *ids, const float *given, const float *g_loss, double *scores, hipStream_t st) {
  const ScoreTable &g = a.g;
  const uint32_t columns = (g.d + 63) / 64, row_columns = o.drows ? columns : 1;
  const uint32_t q_tiles = o.dq ? (g.nq + 15) / 16 * columns : 0, row_tiles = o.drows || o.drow_bias ? (g.n + 15) / 16 * row_columns : 0;
  if (q_tiles + row_tiles == 0) return ANN_OK;
  launch_short<T>(g, scores, st);
  ANN_HIP(hipGetLastError());
  distill_short_weights_kernel<<<(g.nq + 3) / 4, 256, 0, st>>>(g.nq, g.n, scores, k, ids, given, a.lse, g_loss);
  ANN_HIP(hipGetLastError());
  if (g.d % 4 == 0)
    distill_short_grad_kernel<T, kWholePieces><<<q_tiles + row_tiles, 512, 0, st>>>(g, scores, a.lse, o, row_tiles, row_columns, columns);
  else
    distill_short_grad_kernel<T, kShifted><<<q_tiles + row_tiles, 512, 0, st>>>(g, scores, a.lse, o, row_tiles, row_columns, columns);
  ANN_HIP(hipGetLastError());
  return ANN_OK;
}

struct GivenArgs {
  ScoreTable g;
  uint32_t k;
  const uint32_t *ids;
  const float *given, *lse, *g_loss;
  float *whole;     // [nq]: -g T
  uint32_t *rows;   // [nq][k]: the entries' ids; ANN_PAD_ID where none counts
  float *weights;   // [nq][k]: -g t
  uint32_t *slots;  // [n]: filled with ANN_PAD_ID (NULL where not wanted)
};

// Of a query's entries, one to a lane of a wavefront: id (ANN_PAD_ID: it does not count), -g t, and -g T of the query.
struct Entry {
  uint32_t id;
  float weight, whole;
};
__device__ __forceinline__ Entry given_entry(const GivenArgs &a, uint32_t q, uint32_t e) {
  const uint64_t at = (uint64_t)q * a.k + e;
  const bool in = e < a.k, none = a.lse[q] == -INFINITY;
  uint32_t id = in ? a.ids[at] : ANN_PAD_ID;
  const float given = in && id < a.g.n ? a.given[at] : -INFINITY;
  if (given == -INFINITY) id = ANN_PAD_ID;  // (no weight, whatever its row)
  const float g = a.g_loss[q];
  const double t = id < a.g.n ? exp((double)given) : 0.0, all = group_sum_f64<kWave>(t);
  // no row left for this query, the row left out: no gradient
  if (none || (id < a.g.n && a.g.bias && a.g.bias[id] == -INFINITY)) id = ANN_PAD_ID;
  return {id < a.g.n ? id : ANN_PAD_ID, -(float)((double)g * t), none ? 0.0f : -(float)((double)g * all)};
}

// The queries' weights alone, before the power of two that they ask for (f16).
__global__ __launch_bounds__(256) void distill_whole_kernel(GivenArgs a) {
  const uint32_t q = blockIdx.x * 4 + threadIdx.x / kWave;
  if (q >= a.g.nq) return;
  const Entry entry = given_entry(a, q, lane_id());
  if (lane_id() == 0) a.whole[q] = entry.whole;
}

// The entries' weights, and the sum over a query's entries of weight * row: a workgroup to a query (and to each gridDim.y-th part of its columns),
// kGivenLanes pieces of columns at a time, kGivenRuns runs of entries side by side.  T: of the rows.  part NULL: the entries alone.  Workgroups behind
// the queries' only fill the slots.
constexpr uint32_t kGivenRuns = 8, kGivenLanes = 32;
template <typename T, RowEnd END>
__global__ __launch_bounds__(kGivenRuns * kGivenLanes) void distill_more_kernel(GivenArgs a, const float *__restrict__ scaling, float *__restrict__ part) {
  constexpr int VEC = 16 / (int)sizeof(T), kEach = ANN_MAX_ALTERNATIVES / kGivenRuns;
  __shared__ float weight_of[ANN_MAX_ALTERNATIVES], room[kGivenRuns][kGivenLanes * VEC + 4];
  __shared__ uint32_t id_of[ANN_MAX_ALTERNATIVES];
  if (a.slots && blockIdx.y == 0)
    for (uint64_t j = (uint64_t)blockIdx.x * 256 + threadIdx.x; j < a.g.n; j += (uint64_t)gridDim.x * 256) a.slots[j] = ANN_PAD_ID;
  const uint32_t q = blockIdx.x, lane = threadIdx.x % kGivenLanes, run = threadIdx.x / kGivenLanes;
  if (q >= a.g.nq) return;
  const float by = scaling ? scaling[0] : 1.0f;
  if (threadIdx.x < kWave) {
    const uint32_t e = threadIdx.x;
    const uint64_t at = (uint64_t)q * a.k + e;
    const Entry entry = given_entry(a, q, e);
    if (e < a.k && blockIdx.y == 0) a.rows[at] = entry.id, a.weights[at] = entry.weight;
    if (e == 0 && blockIdx.y == 0) a.whole[q] = entry.whole;
    weight_of[e] = entry.weight * by, id_of[e] = entry.id;
  }
  if (!part) return;
  __syncthreads();
  const uint32_t begin = a.k * run / kGivenRuns, end = a.k * (run + 1) / kGivenRuns;
  for (uint32_t c0 = blockIdx.y * (kGivenLanes * VEC); c0 < a.g.d; c0 += gridDim.y * (kGivenLanes * VEC)) {
    const uint32_t c = c0 + lane * VEC;
    RowPiece<T, VEC, END> x[kEach];
#pragma unroll
    for (int u = 0; u < kEach; ++u) {
      const uint32_t id = begin + u < end ? id_of[begin + u] : ANN_PAD_ID;
      x[u].load((const T *)a.g.rows + (id < a.g.n ? id : 0) * a.g.row_stride, id < a.g.n ? c : a.g.d, a.g.d);  // (no row: nothing is read as a number)
    }
    float sum[VEC];
#pragma unroll
    for (int v = 0; v < VEC; ++v) sum[v] = 0.0f;
#pragma unroll
    for (int u = 0; u < kEach; ++u) {
      const uint32_t id = begin + u < end ? id_of[begin + u] : ANN_PAD_ID;
      const float weight = begin + u < end ? weight_of[begin + u] : 0.0f;
#pragma unroll
      for (int v = 0; v < VEC; ++v) sum[v] = id < a.g.n ? __builtin_fmaf(weight, x[u].get(v), sum[v]) : sum[v];
    }
    __syncthreads();  // (the columns before have been read)
#pragma unroll
    for (int v = 0; v < VEC; ++v) room[run][lane * VEC + v] = sum[v];
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < kGivenLanes * VEC && c0 + i < a.g.d; i += kGivenRuns * kGivenLanes) {
      float all = room[0][i];
#pragma unroll
      for (uint32_t r = 1; r < kGivenRuns; ++r) all += room[r][i];
      part[(uint64_t)q * a.g.d + c0 + i] = all;
    }
  }
}

// The second part's sums over the queries, by rows: weights of q, and of the bias.
template <typename T>
struct GivenSums {
  static constexpr bool kWeighted = true, kScalar = true;
  const T *q;
  uint64_t q_stride;
  const float *weights;
  uint32_t *slots;
  float *sums;
  uint32_t k, ld, dim, d;
  bool by_row;  // a sum lies at its row's number; otherwise at that of the run's first entry
  __device__ __forceinline__ const T *row(uint32_t position) const { return q + position / k * q_stride; }
  __device__ __forceinline__ float weight(uint32_t position) const { return weights[position]; }
  __device__ __forceinline__ float scalar(uint32_t position) const { return weights[position]; }
  __device__ __forceinline__ float *at(uint32_t id, uint32_t start) const { return sums + (uint64_t)(by_row ? id : start) * ld; }
  __device__ __forceinline__ void write_scalar(uint32_t id, uint32_t start, float sum) const {
    at(id, start)[d] = sum;
    slots[id] = by_row ? id : start;
  }
  template <int VEC, RowEnd END>
  __device__ __forceinline__ void write(uint32_t id, uint32_t start, uint32_t c, const float (&sum)[VEC]) const {
    float *to = at(id, start) + c;
#pragma unroll
    for (int e = 0; e < VEC; ++e)
      if (VEC == 1 || END == kWholePieces || c + e < dim) to[e] = sum[e];
  }
  __device__ __forceinline__ void beside(uint32_t, uint32_t) const {}
};

struct DistillPlan {
  IdSortPlan sort;
  RunsPlan runs;
  bool by_row = false;
  uint32_t ld = 0;  // of the sums and their parts: d + 1, in pieces of 16 bytes
  uint64_t backward_bytes = 0, whole_at = 0, rows_at = 0, weights_at = 0, scaling_at = 0, slots_at = 0, sort_at = 0, part_at = 0, sums_at = 0;
  Parts parts;
};

// Room for the rows' side is there whether it is wanted or not.
static DistillPlan distill_plan(uint32_t nq, uint64_t n, uint32_t d, uint32_t type, uint32_t k) {
  DistillPlan p;
  if (nq == 0 || n == 0) return p;
  const uint64_t entries = (uint64_t)nq * k;
  p.backward_bytes = scores_backward_bytes(nq, n, d, type, true);
  p.parts.take(p.backward_bytes);
  p.whole_at = p.parts.take(nq * 4ull);
  p.rows_at = p.parts.take(entries * 4), p.weights_at = p.parts.take(entries * 4);
  p.scaling_at = p.parts.take(2 * sizeof(float));
  p.slots_at = p.parts.take(n * 4);
  p.sort = id_sort_plan(entries, n);
  p.sort_at = p.parts.take(p.sort.bytes);
  p.ld = (d + 1 + 3) / 4 * 4;
  p.runs = runs_plan(entries, p.ld);
  p.part_at = p.parts.take(p.runs.part_bytes);
  p.by_row = n <= entries;
  p.sums_at = p.parts.take((p.by_row ? n : entries) * p.ld * sizeof(float));
  return p;
}

template <typename T>
static ann_status distill_rows(const DistillPlan &p, const GivenArgs &a, bool rows, char *ws, GradArgs &to, hipStream_t st) {
  SortedIds sorted;
  if (ann_status s = sort_ids(p.sort, a.rows, ws + p.sort_at, nullptr, NothingBeside(), st, sorted)) return s;
  const uint32_t dim = rows ? a.g.d : 0;
  const Runs runs = {sorted.keys, sorted.positions, a.g.nq * a.k, a.g.n, p.runs.chunk, p.runs.chunks, dim, (float *)(ws + p.part_at), p.ld};
  const GivenSums<T> work = {(const T *)a.g.q, a.g.q_stride, a.weights, a.slots, (float *)(ws + p.sums_at), a.k, p.ld, dim, a.g.d, p.by_row};
  if (ann_status s = sum_runs<T>(runs, work, 0, st)) return s;
  to.slots = a.slots, to.sums = work.sums, to.more_ld = p.ld;
  return ANN_OK;
}

static ann_status check_distillation(const char *what, const ann_row_scores *s, uint32_t k, const uint32_t *ids, const float *given) {
  if (ann_status e = check_scores(what, s)) return e;
  if (k == 0) return fail(ANN_EINVAL, "%s: k == 0", what);
  if (k > ANN_MAX_ALTERNATIVES) return fail(ANN_ECAPACITY, "%s: k = %u exceeds ANN_MAX_ALTERNATIVES = %u", what, k, ANN_MAX_ALTERNATIVES);
  if (s->targets) return fail(ANN_EINVAL, "%s: targets belong to the rows' log probabilities", what);
  if (s->nq && (!ids || !given)) return fail(ANN_EINVAL, "%s: given_ids or given_logprobs is NULL", what);
  return ANN_OK;
}

}  // namespace ann

using namespace ann;

static uint64_t forward_bytes(uint32_t nq, uint64_t n, uint32_t d, uint32_t type) { return (ann_row_logprobs_workspace(nq, n, d, type, 0) + 255) / 256 * 256; }

extern "C" uint64_t ann_row_distillation_workspace(uint32_t nq, uint64_t n, uint32_t d, uint32_t type, uint32_t k) {
  if (n > kMaxRows || nq >= kMaxQueries || d == 0 || type > ANN_BF16 || k > ANN_MAX_ALTERNATIVES || nq == 0) return 0;
  if (short_list(nq, n, d)) return nq * n * sizeof(double);
  return forward_bytes(nq, n, d, type) + nq * 12ull;
}

extern "C" ann_status ann_row_distillation(const ann_row_scores *scores, uint32_t k, const uint32_t *given_ids, const float *given_logprobs, float *loss,
                                           float *lse, float *logprobs, void *workspace, uint64_t workspace_bytes, void *stream) {
  if (ann_status s = check_distillation("ann_row_distillation", scores, k, given_ids, given_logprobs)) return s;
  const uint32_t nq = scores->nq;
  if (nq == 0) return ANN_OK;
  if (!loss || !lse || !logprobs) return fail(ANN_EINVAL, "ann_row_distillation: loss, lse or logprobs is NULL");
  const uint64_t need = ann_row_distillation_workspace(nq, scores->n, scores->d, scores->type, k);
  if (ann_status s = check_workspace("ann_row_distillation", workspace, workspace_bytes, need)) return s;
  const ScoreTable g = score_table(*scores);
  const hipStream_t st = (hipStream_t)stream;
  if (short_list(nq, scores->n, scores->d)) {
    double *all = (double *)workspace;
    if (scores->type == ANN_F32)
      launch_short<float>(g, all, st);
    else if (scores->type == ANN_F16)
      launch_short<f16_t>(g, all, st);
    else
      launch_short<bf16_t>(g, all, st);
    ANN_HIP(hipGetLastError());
    distill_short_loss_kernel<<<(nq + 3) / 4, 256, 0, st>>>(nq, g.n, all, k, given_ids, given_logprobs, loss, lse, logprobs);
    ANN_HIP(hipGetLastError());
    return ANN_OK;
  }
  const uint64_t before = need - nq * 12ull;
  double *wide_lse = (double *)((char *)workspace + before);
  if (ann_status s = row_statistics(*scores, (float *)(wide_lse + nq), lse, wide_lse, workspace, st)) return s;
  if (scores->type == ANN_F32)
    distill_loss_kernel<float><<<nq, 256, 0, st>>>(g, k, given_ids, given_logprobs, wide_lse, loss, logprobs);
  else if (scores->type == ANN_F16)
    distill_loss_kernel<f16_t><<<nq, 256, 0, st>>>(g, k, given_ids, given_logprobs, wide_lse, loss, logprobs);
  else
    distill_loss_kernel<bf16_t><<<nq, 256, 0, st>>>(g, k, given_ids, given_logprobs, wide_lse, loss, logprobs);
  ANN_HIP(hipGetLastError());
  return ANN_OK;
}

extern "C" uint64_t ann_row_distillation_backward_workspace(uint32_t nq, uint64_t n, uint32_t d, uint32_t type, uint32_t k) {
  if (n > kMaxRows || nq >= kMaxQueries || d == 0 || type > ANN_BF16 || k > ANN_MAX_ALTERNATIVES || k == 0) return 0;
  if (short_gradient(nq, n, d)) return nq * n * sizeof(double);
  return distill_plan(nq, n, d, type, k).parts.bytes;
}

extern "C" ann_status ann_row_distillation_backward(const ann_row_scores *scores, uint32_t k, const uint32_t *given_ids, const float *given_logprobs,
                                                    const float *lse, const float *logprobs, const float *g_loss, void *dq, uint64_t dq_stride,
                                                    void *drows, uint64_t drows_stride, float *drow_bias, void *workspace,
                                                    uint64_t workspace_bytes, void *stream) {
  const char *what = "ann_row_distillation_backward";
  if (ann_status s = check_distillation(what, scores, k, given_ids, given_logprobs)) return s;
  if (scores->nq && (!lse || !logprobs || !g_loss)) return fail(ANN_EINVAL, "%s: lse, logprobs or g_loss is NULL", what);
  if (dq && dq_stride < scores->d) return fail(ANN_EINVAL, "%s: dq_stride is shorter than a row", what);
  if (drows && drows_stride < scores->d) return fail(ANN_EINVAL, "%s: drows_stride is shorter than a row", what);
  const uint32_t nq = scores->nq, type = scores->type;
  if (ann_status s = check_workspace(what, workspace, workspace_bytes, ann_row_distillation_backward_workspace(nq, scores->n, scores->d, type, k))) return s;
  char *ws = (char *)workspace;
  const hipStream_t st = (hipStream_t)stream;
  GradArgs a = {};
  a.g = score_table(*scores), a.lse = lse, a.every = true;
  const GradOut o = {dq, drows, drow_bias, dq_stride, drows_stride};
  if (short_gradient(nq, scores->n, scores->d)) {
    double *all = (double *)ws;
    return type == ANN_F32   ? short_backward<float>(a, o, k, given_ids, given_logprobs, g_loss, all, st)
           : type == ANN_F16 ? short_backward<f16_t>(a, o, k, given_ids, given_logprobs, g_loss, all, st)
                             : short_backward<bf16_t>(a, o, k, given_ids, given_logprobs, g_loss, all, st);
  }
  const DistillPlan p = distill_plan(nq, scores->n, scores->d, type, k);
  if (nq && scores->n) {
    const bool rows_side = drows || drow_bias;
    GivenArgs v = {};
    v.g = a.g, v.k = k, v.ids = given_ids, v.given = given_logprobs, v.lse = lse, v.g_loss = g_loss;
    v.whole = (float *)(ws + p.whole_at), v.rows = (uint32_t *)(ws + p.rows_at), v.weights = (float *)(ws + p.weights_at);
    v.slots = rows_side ? (uint32_t *)(ws + p.slots_at) : nullptr;
    const uint32_t filling = rows_side ? (uint32_t)((scores->n + 4095) / 4096 < 2048 ? (scores->n + 4095) / 4096 : 2048) : 0, blocks = nq > filling ? nq : filling;
    a.g_logprob = v.whole;
    float *scaling = nullptr, *part = dq ? scores_backward_more_part(nq, scores->n, scores->d, type, ws) : nullptr;
    if (type == ANN_F16) {
      scaling = (float *)(ws + p.scaling_at);
      distill_whole_kernel<<<(nq + 3) / 4, 256, 0, st>>>(v);
      ANN_HIP(hipGetLastError());
      if (ann_status s = launch_grad_scaling(a, scaling, st)) return s;
      a.scaling = scaling;
    }
    const auto add_up = [&](auto t) {
      typedef decltype(t) T;
      // (few queries: a workgroup to a part of the columns)
      constexpr uint32_t kColumns = kGivenLanes * (16 / sizeof(T));
      const dim3 grid(blocks, part && nq < 256 ? (scores->d + kColumns - 1) / kColumns : 1);
      if (scores->d % (16 / sizeof(T)) == 0)
        distill_more_kernel<T, kWholePieces><<<grid, kGivenRuns * kGivenLanes, 0, st>>>(v, scaling, part);
      else
        distill_more_kernel<T, kShifted><<<grid, kGivenRuns * kGivenLanes, 0, st>>>(v, scaling, part);
    };
    if (type == ANN_F32)
      add_up(0.0f);
    else if (type == ANN_F16)
      add_up(f16_t());
    else
      add_up(bf16_t());
    ANN_HIP(hipGetLastError());
    a.more_part = true;
    if (rows_side) {
      ann_status s = type == ANN_F32   ? distill_rows<float>(p, v, drows, ws, a, st)
                     : type == ANN_F16 ? distill_rows<f16_t>(p, v, drows, ws, a, st)
                                       : distill_rows<bf16_t>(p, v, drows, ws, a, st);
      if (s) return s;
    }
  }
  return scores_backward(type, a, o, ws, st);
}
