// Log probabilities of given rows under the softmax of all rows' scores
// s[i][j] = scale <q_i, x_j> + bias_j, with the softmax' entropy and its largest
// alternatives.  The scores stay in the accumulators of the product: each lane
// keeps, for its queries, a reference m near the largest score, l = sum exp(s - m) and
// t = sum exp(s - m) (s - m) (all fp32) over the rows that pass by; at the end
// lse = m + log l, entropy = log l - t / l.
//
// Without biases (and with a scale that is not negative) m and the exponents are kept times log2 e, so that an exponent is one
// fused multiply-add of the product's result that rounds once: with m in natural units, m log2 e was rounded apart from m, which moved
// all of a lane's exponentials alike (lse, and the log probabilities with it, by up to half a step of 1.44 m).  What the rounding of
// scale log2 e does to lse is made up for at the end, to first order: lse changes by its relative error times the mean score.
//
// Alternatives: the product kernel also writes the largest score of every group of
// rows (one number for kGroup scores).  The k best rows lie in groups whose
// largest score is at least the k-th largest of those; a score may err by what
// score_room() allows, so groups within twice that below it are taken as well,
// and their rows are scored again in fp64 and put in order.  That is exact whatever the
// distribution, ties included; how many rows are scored again is all that depends on it.
// Long rows (more than 128 columns, no stream): a group's second largest score is written as well, and the largest carries
// its row's number in its low four bits; mostly that row alone is scored again (4,000 x 100,003 x 768, k = 20: 400 -> 190 us
// for the end; the product kernel pays 130 of them back).
//
// Three product kernels, chosen by forward_plan(): row_stream_kernel for few queries, bound by reading the rows (1 x 1M x 128 bf16:
// 43 us, 6.0 TB/s; 8 x 200,000 x 960 fp32: 171 us, 4.5 TB/s); row_scores_short_kernel for 16-bit rows of at most 128 columns, bound by the
// instructions of the exponentials (10,000 x 1M x 128: 3.5 ms, 720 TFLOP/s; vector instructions issue in 80 % of the cycles, the matrix cores work in
// 41 %); row_scores_kernel for the rest, bound by the matrix cores' supply (4,000 x 100,003 x 768 without alternatives: 0.84 ms for the call,
// 730 TFLOP/s; the kernel with k = 20: 0.96 ms).
#include "row_logprobs.hpp"

#include <math.h>

namespace ann {

constexpr uint32_t kNormRuns = 2048;    // workgroups that look for the largest row norm: eight to a compute unit
constexpr uint32_t kSplitTarget = 6144; // workgroups of the product kernels for short or few rows: rounds enough to end together
constexpr uint32_t kWideSlots = 512;    // workgroups of the wide product that run at once: two to a compute unit
constexpr float kNothing = -1000.0f;    // an exponent whose power is zero, and finite

// BIAS: natural units; otherwise m and t are times log2 e.
struct Stats {
  float m, l, t;
};
template <bool BIAS>
__device__ __forceinline__ void join(Stats &a, const Stats &b) {
  constexpr float kUnit = BIAS ? kLog2e : 1.0f;
  const float m = fmaxf(a.m, b.m);
  const float da = fmaxf(a.m - m, kNothing), db = fmaxf(b.m - m, kNothing);
  const float fa = __builtin_amdgcn_exp2f(da * kUnit), fb = __builtin_amdgcn_exp2f(db * kUnit);
  a.t = fa * __builtin_fmaf(da, a.l, a.t) + fb * __builtin_fmaf(db, b.l, b.t);
  a.l = __builtin_fmaf(fa, a.l, fb * b.l);
  a.m = m;
}

// A lane's running statistics of one query: l = sum exp(s - m), t = sum exp(s - m) (s - m).  The reference m need not be the
// largest score: it is raised when one lies kSlack above it, which is seldom, and nothing is scaled in between.  (Not further: beside a
// term of e^20 those near one are less than half a step, and t's were lost with them, which count by their exponents; the
// entropy erred by 1.7e-7 of itself with a slack of 20, by 2.2e-8 with this one, its own rounding.)  The scores of a tile are
// summed by themselves and the tiles' sums with what the last addition lost: over a million rows plain sums erred by
// 4.6e-6, ten times the rounding of the scores.
template <bool BIAS>
struct Running {
  static constexpr float kUnit = BIAS ? kLog2e : 1.0f;
  static constexpr float kSlack = BIAS ? 1.5f : 2.0f;
  float m = -3.402823466e38f, l = 0.0f, t = 0.0f, l_lost = 0.0f, t_lost = 0.0f;

  __device__ __forceinline__ bool behind(float top) const { return BIAS ? top > m + kSlack : __builtin_fmaf(top, kLog2e, -m) > kSlack; }
  __device__ __forceinline__ void raise(float top) {
    const float next = behind(top) ? BIAS ? top : top * kLog2e : m, step = fmaxf(m - next, kNothing), f = __builtin_amdgcn_exp2f(step * kUnit);
    t = f * __builtin_fmaf(step, l, t), t_lost *= f;
    l *= f, l_lost *= f;
    m = next;
  }
  static __device__ __forceinline__ void add(float &sum, float &lost, float v) {
    v -= lost;
    const float next = sum + v;
    lost = (next - sum) - v;
    sum = next;
  }
  // N scores, none of which lies far above m: whole ones with BIAS, else they are s * scale, with c = scale log2 e.  MASKED: -infinity
  // means a row left out.
  template <bool MASKED, int N>
  __device__ __forceinline__ void take(const float (&s)[N], float c) {
    float sum = 0.0f, weighed = 0.0f;
#pragma unroll
    for (int r = 0; r < N; ++r) {
      float y = BIAS ? s[r] - m : __builtin_fmaf(s[r], c, -m);
      if (MASKED) y = s[r] == -INFINITY ? kNothing : y;
      const float p = __builtin_amdgcn_exp2f(y * kUnit);
      sum += p;
      weighed = __builtin_fmaf(p, y, weighed);
    }
    add(l, l_lost, sum);
    add(t, t_lost, weighed);
  }
  __device__ __forceinline__ Stats stats() const { return {m, l, t}; }
};

// Rows of a group of 64: a wavefront's of a tile.  Of a group of 16: those of one half of the lanes in a block of 32.
__host__ __device__ constexpr uint32_t group_count(uint32_t n, int group) { return group == 64 ? (n + 63) / 64 : (n + 31) / 32 * 2; }

// Where a query's groups lie from the one's before (groups of 16: so that eight of them are two aligned pieces of 16 bytes).
__host__ __device__ constexpr uint32_t group_stride(uint32_t n, int group) { return group == 64 ? group_count(n, 64) : (group_count(n, 16) + 7) / 8 * 8; }

// A block of 32 rows x 32 queries, rows down the registers and queries along the lanes.  BIAS: scores are made whole, bias[32] (LDS)
// added.  MASKED: -infinity where a row does not count.  Then the lane's largest score (of 16 rows).
template <bool MASKED, bool BIAS>
__device__ __forceinline__ void add_bias(f32x16 &acc, const float *bias, float scale) {
  static_assert(MASKED || !BIAS, "biases may leave rows out");
  if constexpr (MASKED) {
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const float b = bias[block_row(r)];
      acc[r] = b == -INFINITY ? -INFINITY : BIAS ? __builtin_fmaf(acc[r], scale, b) : acc[r];
    }
  }
}
// The score of a largest element (a scale of zero leaves -infinity, no row at all, as it is).
template <bool MASKED, bool BIAS>
__device__ __forceinline__ float scaled(float top, float scale) {
  return BIAS || (MASKED && top == -INFINITY) ? top : top * scale;
}
template <bool MASKED, bool BIAS>
__device__ __forceinline__ float largest_of(const f32x16 &acc, float scale) {
  float top = acc[0];
#pragma unroll
  for (int r = 1; r < 16; ++r) top = fmaxf(top, acc[r]);
  return scaled<MASKED, BIAS>(top, scale);
}
// The largest of the lane's 16 scores, its low four bits replaced by its number, and the second largest.  (Infinite scores stand for the
// lowest and the largest number: they have no bits to spare.  Without biases they come with rows whose norm is infinite, and then the
// maxima are not used.)
struct TopTwo {
  float first, second;
};
__device__ __forceinline__ float numbered(float s, uint32_t r) { return __uint_as_float((__float_as_uint(s) & ~15u) | r); }
__device__ __forceinline__ float finite(float s) { return __builtin_amdgcn_fmed3f(s, -3.402823466e38f, 3.402823466e38f); }
template <bool MASKED, bool BIAS>
__device__ __forceinline__ TopTwo two_largest_of(const f32x16 &acc, float scale) {
  TopTwo t = {-3.402823466e38f, -3.402823466e38f};
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    const float s = numbered(MASKED ? finite(acc[r]) : acc[r], r);
    t.second = r ? fmaxf(t.second, fminf(t.first, s)) : t.second;
    t.first = r ? fmaxf(t.first, s) : s;
  }
  if constexpr (!BIAS) {
    const float first = t.first * scale;
    t = {numbered(MASKED ? finite(first) : first, __float_as_uint(t.first) & 15u), t.second * scale};
  }
  return t;
}
template <bool MASKED, bool BIAS>
__device__ __forceinline__ void take_block(const f32x16 &acc, Running<BIAS> &run, float c) {
  float s[16];
#pragma unroll
  for (int r = 0; r < 16; ++r) s[r] = acc[r];
  run.template take<MASKED>(s, c);
}

// Writes the largest scores of the groups of 64 rows from row0, of which the lane has seen the halves of two blocks.
template <int GROUP>
__device__ __forceinline__ void put_groups(float top0, float top1, uint32_t q, uint32_t nq, uint32_t row0, uint32_t n_groups, uint32_t stride, float *__restrict__ group_max) {
  const int lane = lane_id();
  float *out = group_max + (uint64_t)q * stride;
  if constexpr (GROUP == 64) {
    const LanePair p = lane_pair<false>(__float_as_uint(fmaxf(top0, top1)));
    const float all = fmaxf(__uint_as_float(p.low), __uint_as_float(p.high));
    if (lane < 32 && q < nq && row0 / 64 < n_groups) out[row0 / 64] = all;
  } else if constexpr (GROUP == 16) {
    const uint32_t at = row0 / 16 + lane / 32;
    if (q < nq && at < n_groups) out[at] = top0;
    if (q < nq && at + 2 < n_groups) out[at + 2] = top1;
  }
}

// The statistics of the two lanes, 32 apart, that share a query.
template <bool BIAS>
__device__ __forceinline__ Stats join_halves(const Stats &s) {
  const LanePair m = lane_pair<false>(__float_as_uint(s.m)), l = lane_pair<false>(__float_as_uint(s.l)), t = lane_pair<false>(__float_as_uint(s.t));
  Stats a = {__uint_as_float(m.low), __uint_as_float(l.low), __uint_as_float(t.low)};
  join<BIAS>(a, {__uint_as_float(m.high), __uint_as_float(l.high), __uint_as_float(t.high)});
  return a;
}

// BIAS: rows may be left out, or the scale is negative.  MB: blocks of 32 rows to a wavefront; four: the wide product, for 16-bit
// rows of whole slices where tiles of 256 rows still fill the card (4,000 x 100,003 x 768 fp16, the call: 1,074 us against 1,118 by tiles of 128 with
// k = 20, 840 against 922 without alternatives, though 29 registers a lane are kept in scratch memory).
// APART (fp32): the smaller products of parts are summed apart.
template <typename T, bool BIAS, int GROUP, int MB, bool APART = false>
__global__ __launch_bounds__(256, MB == 4 ? 2 : 1) void row_scores_kernel(ScoreTable g, uint32_t q_tiles, uint32_t q_group, uint32_t splits, float4 *__restrict__ stats,
                                                         float *__restrict__ group_max, float *__restrict__ group_second) {
  constexpr int kMore = MB == 4 ? kWideBuffer : 16;
  __shared__ __attribute__((aligned(16))) char lds[MB == 4 ? kWideBuffer : kTileBytes<T, kAlong, kAlong>], lds1[kMore], lds2[kMore];
  __shared__ float row_bias[MB * 64];
  constexpr uint32_t kRowTile = MB * 64;
  // Workgroup b runs on die b mod 8.  A die takes a run of the pairs of a group of query tiles and a split of the rows, the queries of a
  // group next to each other: these stay in its L2 (all queries of 4,096 x 768 are more than it holds, and the product waited
  // for them), and every tile of rows is read by a group at a time.
  const uint32_t groups = (q_tiles + q_group - 1) / q_group, pairs = groups * splits, per_die = (pairs + 7) / 8;
  const uint32_t b8 = blockIdx.x / 8, in_die = b8 / q_group, pair = blockIdx.x % 8 * per_die + in_die;
  const uint32_t qt = pair / splits * q_group + b8 % q_group, split = pair % splits;
  if (in_die >= per_die || pair >= pairs || qt >= q_tiles) return;
  const uint32_t row_tiles = (g.n + kRowTile - 1) / kRowTile;
  const uint32_t first = (uint32_t)((uint64_t)row_tiles * split / splits), last = (uint32_t)((uint64_t)row_tiles * (split + 1) / splits);
  const int wave = (int)threadIdx.x / kWave, lane = lane_id(), mw = wave / 2 * MB * 32, nw = wave % 2 * 64;
  const Lines<T> X = {(const T *)g.rows, g.row_stride, g.n, g.d}, Q = {(const T *)g.q, g.q_stride, g.nq, g.d};
  const uint32_t n_groups = GROUP ? group_count(g.n, GROUP) : 0, stride = GROUP ? group_stride(g.n, GROUP) : 0;
  const float c = g.scale * kLog2e;
  Running<BIAS> run[2];
  for (uint32_t tile = first; tile < last; ++tile) {
    const uint32_t row0 = tile * kRowTile;
    const bool whole = row0 + kRowTile <= g.n;
    f32x16 acc[MB][2];
    clear(acc);
    if constexpr (MB == 4)
      wide_product<T, kAlong, kAlong>(acc, X, row0, Q, qt * kTile, 0, g.d, lds, lds1, lds2);
    else
      // (fp32: the smaller products apart take so many registers that one workgroup fits where two did: 155 -> 213 us for 513 x 50,000 x 100;
      // with one sum the log probabilities err by 6e-8 there, by 2.8e-7 with 768 columns, about as far as a plain fp32 product's.  Distillation, whose
      // losses are differences of them, has them apart: 105 -> 167 us for that size, 690 -> 1,010 for 4,096 x 100,000 x 128)
      tile_product<T, kAlong, kAlong, APART>(acc, X, row0, Q, qt * kTile, 0, g.d, lds);
    if (BIAS || !whole) {
      // (read by the tile before's epilogue: the barriers of the product lie in between; d > 0)
      if (threadIdx.x < kRowTile) row_bias[threadIdx.x] = row0 + threadIdx.x < g.n ? (BIAS && g.bias ? g.bias[row0 + threadIdx.x] : 0.0f) : -INFINITY;
      __syncthreads();
    }
    const auto finish = [&](auto masked) {
      constexpr bool MASKED = decltype(masked)::value;
      const bool is_numbered = GROUP == 16 && (MB == 4 || group_second);
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const uint32_t q = qt * kTile + nw + j * 32 + lane % 32;
        // (two blocks at a time, each with a look at the reference: no more intermediate values are live than fit)
#pragma unroll
        for (int i0 = 0; i0 < MB; i0 += 2) {
          float top[2], second[2];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            f32x16 &block = acc[i0 + i][j];
            add_bias<MASKED, BIAS>(block, row_bias + mw + (i0 + i) * 32, g.scale);
            if (is_numbered) {
              const TopTwo t = two_largest_of<MASKED, BIAS>(block, g.scale);
              top[i] = t.first, second[i] = t.second;
            } else {
              top[i] = largest_of<MASKED, BIAS>(block, g.scale);
            }
            if (__any(run[j].behind(top[i]))) run[j].raise(top[i]);
            take_block<MASKED, BIAS>(block, run[j], c);
            if (MB == 4) __builtin_amdgcn_sched_barrier(0);
          }
          put_groups<GROUP>(top[0], top[1], q, g.nq, row0 + mw + i0 * 32, n_groups, stride, group_max);
          if (is_numbered) put_groups<GROUP>(second[0], second[1], q, g.nq, row0 + mw + i0 * 32, n_groups, stride, group_second);
        }
      }
    };
    if (BIAS || !whole)
      finish(std::true_type());
    else
      finish(std::integral_constant<bool, BIAS>());
  }
  // the two halves of a wavefront, then the two wavefronts that share queries
  __shared__ Stats other[2][64];
  Stats st[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    st[j] = join_halves<BIAS>(run[j].stats());
    if (wave >= 2 && lane < 32) other[wave % 2][j * 32 + lane] = st[j];
  }
  __syncthreads();
  if (wave < 2 && lane < 32) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      join<BIAS>(st[j], other[wave][j * 32 + lane]);
      const uint32_t q = qt * kTile + nw + j * 32 + lane;
      if (q < g.nq) stats[(uint64_t)split * g.nq + q] = make_float4(st[j].m, st[j].l, st[j].t, 0.0f);
    }
  }
}

// Short rows of 16 bits, KS slices of 16 columns: the queries stay in registers, as the matrix instruction takes them, 64 to a
// wavefront, and tiles of 64 rows pass by in LDS.  With 128 columns a score costs 256 operations on the matrix cores and
// an exponential with four more instructions, so the end of a block counts as much as its product: the product of a block of 32 rows and
// the end of the one before it are one stretch of code, so that the matrix cores work meanwhile.  What is left is bound by the
// instructions of the end, so addresses are kept cheap: lines of LDS are 16 bytes apart from a power of two (eight
// lines read side by side hit all banks, and every piece lies at a constant distance), and offsets within a tile are 32 bits.
constexpr int kShortRows = 64, kShortQueries = 256;
constexpr uint64_t kShortStride = 1u << 24;  // longest row stride

template <typename T, int KS, bool BIAS, int GROUP>
__global__ __launch_bounds__(256, 2) void row_scores_short_kernel(ScoreTable g, uint32_t q_tiles, uint32_t splits, float4 *__restrict__ stats,
                                                                  float *__restrict__ group_max) {
  typedef typename Operand16<T>::E E;
  constexpr int kSlots = 2 * KS, kLine = KS * 32 + 16, kUnits = (kShortRows * kSlots + 255) / 256;
  __shared__ __attribute__((aligned(16))) char lds[2][kShortRows * kLine];
  __shared__ float row_bias[4][kShortRows];  // (of a tile: written while some wavefront may still read that of two tiles before)
  // workgroup b runs on die b mod 8: a die takes all queries through its own part of the rows
  const uint32_t b8 = blockIdx.x / 8, qt = b8 % q_tiles, split = b8 / q_tiles * 8 + blockIdx.x % 8;
  if (split >= splits) return;
  const uint32_t tiles = (g.n + kShortRows - 1) / kShortRows;
  const uint32_t first = (uint32_t)((uint64_t)tiles * split / splits), last = (uint32_t)((uint64_t)tiles * (split + 1) / splits);
  const int wave = (int)threadIdx.x / kWave, lane = lane_id();
  const T *rows = (const T *)g.rows;
  const uint32_t n_groups = GROUP ? group_count(g.n, GROUP) : 0, stride = GROUP ? group_stride(g.n, GROUP) : 0, q = qt * kShortQueries + wave * 64 + lane % 32;  // (and q + 32)
  const float c = g.scale * kLog2e;
  E query[2][KS];
#pragma unroll
  for (int j = 0; j < 2; ++j)
#pragma unroll
    for (int kk = 0; kk < KS; ++kk) {
      const uint32_t k = kk * 16 + lane / 32 * 8;
      Unit<T> u;
      load_unit(u, (const T *)g.q + (q + j * 32) * g.q_stride + k, q + j * 32 < g.nq ? (int64_t)g.d - k : 0);
      query[j][kk] = __builtin_bit_cast(E, u);
    }
  Unit<T> u[kUnits];
  uint32_t from[kUnits], to[kUnits];
#pragma unroll
  for (int i = 0; i < kUnits; ++i) {
    const uint32_t at = threadIdx.x + 256 * i, line = at / kSlots, slot = at % kSlots;
    from[i] = (line * (uint32_t)g.row_stride + slot * 8) * sizeof(T);
    to[i] = line * kLine + slot * 16;
  }
  constexpr bool kEven = kUnits * 256 == kShortRows * kSlots;  // every lane has as many units
  const auto fetch = [&](uint32_t tile) {
    const char *base = (const char *)(rows + (uint64_t)tile * kShortRows * g.row_stride);
    if (KS * 16 == g.d && (tile + 1) * kShortRows <= g.n) {
#pragma unroll
      for (int i = 0; i < kUnits; ++i)
        if (kEven || threadIdx.x + 256 * i < kShortRows * kSlots) load_unit(u[i], (const T *)(base + from[i]));
    } else {
#pragma unroll
      for (int i = 0; i < kUnits; ++i) {
        const uint32_t at = threadIdx.x + 256 * i, row = tile * kShortRows + at / kSlots, k = at % kSlots * 8;
        if (kEven || at < kShortRows * kSlots) load_unit(u[i], (const T *)(base + from[i]), row < g.n ? (int64_t)g.d - k : 0);
      }
    }
  };
  // Tile into LDS, the next one on its way.  (One barrier per tile: whoever writes this half again has met the others at the next tile's.)
  const auto enter = [&](uint32_t tile) {
    char *at = lds[tile & 1];
#pragma unroll
    for (int i = 0; i < kUnits; ++i)
      if (kEven || threadIdx.x + 256 * i < kShortRows * kSlots) *(uint4 *)(at + to[i]) = unit_part(u[i], 0);
    const uint32_t row = tile * kShortRows + threadIdx.x;
    if ((BIAS || tile * kShortRows + kShortRows > g.n) && threadIdx.x < kShortRows)
      row_bias[tile & 3][threadIdx.x] = row < g.n ? (BIAS && g.bias ? g.bias[row] : 0.0f) : -INFINITY;
    __syncthreads();
    if (tile + 1 < last) fetch(tile + 1);
  };
  const auto product = [&](f32x16(&acc)[2], uint32_t tile, int half) {
    const char *at = lds[tile & 1] + lane % 32 * kLine + lane / 32 * 16;
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[j][r] = 0.0f;
#pragma unroll
    for (int kk = 0; kk < KS; ++kk) {
      const E x = *(const E *)(at + half * 32 * kLine + kk * 32);
#pragma unroll
      for (int j = 0; j < 2; ++j) acc[j] = matrix_step(x, query[j][kk], acc[j]);
    }
  };
  Running<BIAS> run[2];
  float top[2][2];  // of either half of a tile
  // The scores of a half of a tile are taken on while `also` (the next half's product) is formed.
  const auto end = [&](f32x16(&past)[2], uint32_t tile, int half, auto also) {
    const auto with = [&](auto masked) {
      constexpr bool MASKED = decltype(masked)::value;
      bool behind = false;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        add_bias<MASKED, BIAS>(past[j], row_bias[tile & 3] + half * 32, g.scale);
        top[half][j] = largest_of<MASKED, BIAS>(past[j], g.scale);
        behind |= run[j].behind(top[half][j]);
      }
      if (__any(behind)) {
#pragma unroll
        for (int j = 0; j < 2; ++j) run[j].raise(top[half][j]);
      }
      also();
#pragma unroll
      for (int j = 0; j < 2; ++j) take_block<MASKED, BIAS>(past[j], run[j], c);
    };
    if (BIAS || tile * kShortRows + kShortRows > g.n)
      with(std::true_type());
    else
      with(std::integral_constant<bool, BIAS>());
    if (GROUP != 0 && half) {
#pragma unroll
      for (int j = 0; j < 2; ++j) put_groups<GROUP>(top[0][j], top[1][j], q + j * 32, g.nq, tile * kShortRows, n_groups, stride, group_max);
    }
  };
  if (first < last) {
    f32x16 upper[2], lower[2];
    fetch(first);
    enter(first);
    product(upper, first, 0);
    for (uint32_t tile = first; tile < last; ++tile) {
      end(upper, tile, 0, [&] { product(lower, tile, 1); });
      if (tile + 1 < last) {
        enter(tile + 1);
        end(lower, tile, 1, [&] { product(upper, tile + 1, 0); });
      } else {
        end(lower, tile, 1, [] {});
      }
    }
  }
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const Stats s = join_halves<BIAS>(run[j].stats());
    if (lane < 32 && q + j * 32 < g.nq) stats[(uint64_t)split * g.nq + q + j * 32] = make_float4(s.m, s.l, s.t, 0.0f);
  }
}

// Few queries: the rows are read once, straight into registers, and multiplied by blocks of 16 queries that
// wait in LDS as the 16x16x32 instruction takes them.  Bound by reading the rows.  A wavefront takes 64 rows at a time, four
// blocks of 16, and kSteps slices of 32 columns of them per round; the next round's are on their way meanwhile.  Row m of block b
// of a pair is row 8 (m / 4) + 4 b + m % 4 of the pair's 32, so that blocks are the same groups of 16 as above.  The rows' norms
// (for score_room) are summed on the way.
constexpr int kStreamThreads = 512;
constexpr int kStreamRows = 64;         // to a wavefront at a time
constexpr uint32_t kStreamGroups = 256; // workgroups: one to a compute unit, eight wavefronts each
constexpr uint32_t kStreamLds = 152u << 10;  // of the 160 KiB, for queries

typedef float f32x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ f32x4 small_step(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 small_step(f16x8 a, f16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

__device__ __forceinline__ float add_squares(const Unit<bf16_t> &u, float sum) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    const bf16x2 v = {u.v[e], u.v[e + 1]};
    sum = __builtin_amdgcn_fdot2_f32_bf16(v, v, sum, false);
  }
  return sum;
}
__device__ __forceinline__ float add_squares(const Unit<f16_t> &u, float sum) {
  typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    const f16x2 v = {u.v[e], u.v[e + 1]};
    sum = __builtin_amdgcn_fdot2(v, v, sum, false);
  }
  return sum;
}
__device__ __forceinline__ float add_squares(const Unit<float> &u, float sum) {
#pragma unroll
  for (int e = 0; e < 8; ++e) sum = __builtin_fmaf(u.v[e], u.v[e], sum);
  return sum;
}

template <typename T>
constexpr int kSteps = sizeof(T) == 4 ? 2 : 4;  // 64 registers of rows on their way

// NB: blocks of 16 queries.
template <typename T, int NB, bool BIAS, int GROUP>
__global__ __launch_bounds__(kStreamThreads) void row_stream_kernel(ScoreTable g, float4 *__restrict__ stats, float *__restrict__ group_max,
                                                                    float *__restrict__ norms) {
  typedef Operand16<T> O;
  typedef typename O::E E;
  constexpr int kWaves = kStreamThreads / kWave, S = kSteps<T>;
  extern __shared__ __attribute__((aligned(16))) char dynamic[];  // [steps][parts][NB] pieces of 64 lanes x 16 bytes; later the wavefronts' statistics
  const uint32_t steps = (g.d + 31) / 32, rounds = (steps + S - 1) / S;
  const int lane = lane_id(), wave = (int)threadIdx.x / kWave, part = lane / 16;
  for (uint32_t at = threadIdx.x; at < steps * NB * 64; at += kStreamThreads) {
    const uint32_t q = at / 64 % NB * 16 + at % 16, step = at / (64 * NB), k = step * 32 + at % 64 / 16 * 8;
    Unit<T> u;
    load_unit(u, (const T *)g.q + q * g.q_stride + k, q < g.nq ? (int64_t)g.d - k : 0);
#pragma unroll
    for (int p = 0; p < O::kParts; ++p) *(uint4 *)(dynamic + (((uint64_t)step * O::kParts + p) * NB * 64 + at % (64 * NB)) * 16) = unit_part(u, p);
  }
  __syncthreads();
  // blocks of 64 rows in turn to the wavefronts of the workgroup, which has a run of them to itself
  const uint32_t blocks = (g.n + kStreamRows - 1) / kStreamRows;
  const uint32_t first = (uint32_t)((uint64_t)blocks * blockIdx.x / gridDim.x), last = (uint32_t)((uint64_t)blocks * (blockIdx.x + 1) / gridDim.x);
  const uint32_t n_groups = GROUP ? group_count(g.n, GROUP) : 0, stride = GROUP ? group_stride(g.n, GROUP) : 0;
  const float c = g.scale * kLog2e;
  const T *rows = (const T *)g.rows;
  const int in_block = lane % 16 / 4 * 8 + lane % 4;  // the lane's row of a pair's 32, of its first block
  Unit<T> now[S][4], next[S][4];
  // (rows behind the last are the last once more: they do not count; slices behind the last are not used)
  const auto fetch = [&](Unit<T>(&u)[S][4], uint32_t block, uint32_t round) {
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      uint32_t row = block * kStreamRows + b / 2 * 32 + b % 2 * 4 + in_block;
      row = row < g.n ? row : g.n - 1;
      const T *x = rows + row * g.row_stride;
#pragma unroll
      for (int s = 0; s < S; ++s) {
        const uint32_t k = (round * S + s) * 32 + part * 8;
        if ((round * S + s + 1) * 32 <= g.d)
          load_unit(u[s][b], x + k, 8);
        else
          load_unit(u[s][b], x + k, (int64_t)g.d - k);
      }
    }
  };
  Running<BIAS> run[NB];
  constexpr bool kApart = O::kParts > 1;
  f32x4 acc[NB][4], low[kApart ? NB : 1][4];  // low: the smaller products of fp32 parts, so that the sum rounds once per 32 columns and not six times
  float squares[4] = {0.0f, 0.0f, 0.0f, 0.0f}, largest = 0.0f;
  uint32_t block = first + wave, round = 0;
  if (block < last) fetch(next, block, 0);
  while (block < last) {
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
      for (int b = 0; b < 4; ++b) now[s][b] = next[s][b];
    const bool ends = round + 1 == rounds;
    const uint32_t next_block = ends ? block + kWaves : block, next_round = ends ? 0 : round + 1;
    if (next_block < last) fetch(next, next_block, next_round);
    if (round == 0) {
#pragma unroll
      for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          acc[j][b] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
          if constexpr (kApart) low[j][b] = acc[j][b];
        }
    }
#pragma unroll
    for (int s = 0; s < S; ++s) {
      if (round * S + s >= steps) break;
      E q[O::kParts][NB];
      const char *at = dynamic + (uint64_t)(round * S + s) * O::kParts * NB * 1024 + lane * 16;
#pragma unroll
      for (int p = 0; p < O::kParts; ++p)
#pragma unroll
        for (int j = 0; j < NB; ++j) q[p][j] = *(const E *)(at + (p * NB + j) * 1024);
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        if constexpr (GROUP != 0) squares[b] = add_squares(now[s][b], squares[b]);
        E x[O::kParts];
#pragma unroll
        for (int p = 0; p < O::kParts; ++p) x[p] = __builtin_bit_cast(E, unit_part(now[s][b], p));
#pragma unroll
        for (int sum = O::kParts - 1; sum >= 0; --sum)
#pragma unroll
          for (int p = 0; p <= sum; ++p)
#pragma unroll
            for (int j = 0; j < NB; ++j) {
              f32x4 &to = kApart && sum != 0 ? low[kApart ? j : 0][b] : acc[j][b];
              to = small_step(x[p], q[sum - p][j], to);
            }
      }
    }
    if (ends) {
      const uint32_t row0 = block * kStreamRows;
      const bool whole = row0 + kStreamRows <= g.n;
      if constexpr (GROUP != 0) {
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          const uint32_t row = row0 + b / 2 * 32 + b % 2 * 4 + in_block;
          const bool out = BIAS && g.bias && row < g.n && g.bias[row] == -INFINITY;
          if (!out) largest = fmaxf(largest, squares[b]);
          squares[b] = 0.0f;
        }
      }
      float bias[16];
      if (BIAS || !whole) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const uint32_t row = row0 + r / 8 * 32 + part * 8 + r % 8;  // (r / 4: the block)
          bias[r] = row < g.n ? (BIAS && g.bias ? g.bias[row] : 0.0f) : -INFINITY;
        }
      }
      const auto finish = [&](auto masked) {
        constexpr bool MASKED = decltype(masked)::value;
#pragma unroll
        for (int j = 0; j < NB; ++j) {
          float s[16], top[4];
#pragma unroll
          for (int b = 0; b < 4; ++b) {
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const int i = b * 4 + r;
              s[i] = kApart ? acc[j][b][r] + low[kApart ? j : 0][b][r] : acc[j][b][r];
              if constexpr (MASKED) s[i] = bias[i] == -INFINITY ? -INFINITY : BIAS ? __builtin_fmaf(s[i], g.scale, bias[i]) : s[i];
              top[b] = r ? fmaxf(top[b], s[i]) : s[i];
            }
            top[b] = scaled<MASKED, BIAS>(top[b], g.scale);
          }
          const float all = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
          if constexpr (GROUP != 0) {
            const uint32_t q = j * 16 + lane % 16;
            const auto over_parts = [](float v) {  // the other lanes' of the same query
              LanePair p = lane_pair<true>(__float_as_uint(v));
              v = fmaxf(__uint_as_float(p.low), __uint_as_float(p.high));
              p = lane_pair<false>(__float_as_uint(v));
              return fmaxf(__uint_as_float(p.low), __uint_as_float(p.high));
            };
            float *out = group_max + (uint64_t)q * stride;
            if constexpr (GROUP == 64) {
              const float most = over_parts(all);
              if (lane < 16 && q < g.nq) out[block] = most;
            } else {
#pragma unroll
              for (int b = 0; b < 4; ++b) {
                const float most = over_parts(top[b]);
                if (part == b && q < g.nq && block * 4 + b < n_groups) out[block * 4 + b] = most;
              }
            }
          }
          if (__any(run[j].behind(all))) run[j].raise(all);
          run[j].template take<MASKED>(s, c);
        }
      };
      if (BIAS || !whole)
        finish(std::true_type());
      else
        finish(std::integral_constant<bool, BIAS>());
    }
    block = next_block, round = next_round;
  }
  // lanes that share a query, then wavefronts
  __syncthreads();
  Stats *room = (Stats *)dynamic;  // [kWaves][NB * 16]
#pragma unroll
  for (int j = 0; j < NB; ++j) {
    Stats a = run[j].stats();
#pragma unroll
    for (int far = 16; far < 64; far *= 2) {
      const Stats b = {__int_as_float(xor_lane_i32(__float_as_int(a.m), far)), __int_as_float(xor_lane_i32(__float_as_int(a.l), far)),
                       __int_as_float(xor_lane_i32(__float_as_int(a.t), far))};
      join<BIAS>(a, b);
    }
    if (lane < 16) room[wave * NB * 16 + j * 16 + lane] = a;
  }
  __shared__ float most[kWaves];
  if constexpr (GROUP != 0) {
    // a row's norm is the sum of its four lanes' shares, at most the sum of their largest
    float v = largest;
    v = fmaxf(v, __int_as_float(dpp_i32<kDppQuadXor1>(__float_as_int(v))));
    v = fmaxf(v, __int_as_float(dpp_i32<kDppQuadXor2>(__float_as_int(v))));
    v = fmaxf(v, __int_as_float(dpp_i32<kDppRowHalfMirror>(__float_as_int(v))));
    v = fmaxf(v, __int_as_float(dpp_i32<kDppRowMirror>(__float_as_int(v))));
    LanePair p = lane_pair<true>(__float_as_uint(v));
    v = __uint_as_float(p.low) + __uint_as_float(p.high);
    p = lane_pair<false>(__float_as_uint(v));
    v = __uint_as_float(p.low) + __uint_as_float(p.high);
    if (lane == 0) most[wave] = v;
  }
  __syncthreads();
  if (threadIdx.x < NB * 16 && threadIdx.x < g.nq) {
    Stats a = room[threadIdx.x];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) join<BIAS>(a, room[w * NB * 16 + threadIdx.x]);
    stats[(uint64_t)blockIdx.x * g.nq + threadIdx.x] = make_float4(a.m, a.l, a.t, 0.0f);
  }
  if (GROUP != 0 && threadIdx.x == 0) {
    float v = most[0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) v = fmaxf(v, most[w]);
    norms[blockIdx.x] = v;
  }
}

// The largest squared norm of the rows of each workgroup that are not left out (for the error of a score; NaN: of no
// interest, such a row is no alternative).
template <typename T>
__global__ __launch_bounds__(256) void row_norms_kernel(ScoreTable g, float *__restrict__ out) {
  __shared__ float room[4];
  const uint32_t lane = threadIdx.x % 16;
  float most = 0.0f;
  for (uint64_t row = blockIdx.x * 16ull + threadIdx.x / 16; row < g.n; row += gridDim.x * 16ull) {
    const T *x = (const T *)g.rows + row * g.row_stride;
    float sum = 0.0f;
    for (uint32_t k = lane * 8; k < g.d; k += 128) {
      Unit<T> u;
      load_unit(u, x + k, (int64_t)g.d - k);
#pragma unroll
      for (int e = 0; e < 8; ++e) sum = __builtin_fmaf(to_f32(u.v[e]), to_f32(u.v[e]), sum);
    }
    sum += __int_as_float(dpp_i32<kDppQuadXor1>(__float_as_int(sum)));
    sum += __int_as_float(dpp_i32<kDppQuadXor2>(__float_as_int(sum)));
    sum += __int_as_float(dpp_i32<kDppRowHalfMirror>(__float_as_int(sum)));
    sum += __int_as_float(dpp_i32<kDppRowMirror>(__float_as_int(sum)));
    if (!(g.bias && g.bias[row] == -INFINITY)) most = fmaxf(most, sum);
  }
  most = wave_max_f32(most);
  if (threadIdx.x % kWave == 0) room[threadIdx.x / kWave] = most;
  __syncthreads();
  if (threadIdx.x == 0) out[blockIdx.x] = fmaxf(fmaxf(room[0], room[1]), fmaxf(room[2], room[3]));
}

// How far a score of the product kernel may lie from its value: each of d additions rounds a
// partial sum of at most |q| |x| (2^-24 of it; twice that for the order inside the
// instruction), the products of parts left out are below 2^-23 of |q| |x|, and the last
// product and addition round a score, which is at most `largest` in size.  fp32: six products to an element.
// Below fp32's normal numbers roundings are steps of their own size (a number in the low four bits is up to 16 of
// the smallest), and products and parts may be taken for zero: at most 2^-126 to an addition, before and after the scale.
__device__ __forceinline__ float score_room(uint32_t d, bool parts, bool is_numbered, float q_norm, float x_norm, float scale, float largest) {
  const float size = fabsf(scale) * q_norm * x_norm * 1.001f;
  const float additions = (parts ? 6.0f : 1.0f) * (float)d + 64.0f;
  return additions * 0x1p-23f * size + (is_numbered ? 0x1p-18f : 0x1p-22f) * (largest + size) + additions * 0x1p-126f * (1.0f + fabsf(scale));
}

constexpr uint32_t kListed = 1024;      // groups that are taken up at a time
constexpr uint32_t kBest = 512;         // scored candidates that are kept at a time
constexpr uint32_t kFewQueries = 512;   // fewer get a workgroup of 1,024 lanes each
constexpr uint32_t kInFlight = 8;       // groups' scores that a lane reads at once
constexpr uint32_t kTops = 256;         // largest scores of so many parts of the groups bound the k-th

struct FinishArgs {
  ScoreTable g;
  const uint32_t *targets;
  const float4 *stats;
  const float *group_max, *group_second, *norms;  // group_second: with numbered largest scores (groups of 16), else NULL
  uint32_t splits, k, norm_runs;
  double unit, scale_error;  // natural units to one of the statistics'; how much scale log2 e lacks where the kernels take it rounded, relative
  float *logprob, *entropy, *lse, *alt_logprobs;
  uint32_t *alt_ids;
  double *wide_lse;  // before it is rounded (NULL where not wanted)
};

// A row's product with the query (in LDS, zero from d on) in fp64, by LANES lanes.
template <typename T, int LANES>
__device__ __forceinline__ double exact_dot(const T *x, const float *q, uint32_t d) {
  double sum = 0.0;
  for (uint32_t k = lane_id() % LANES * 8; k < d; k += LANES * 8) {
    Unit<T> u;
    load_unit(u, x + k, (int64_t)d - k);
#pragma unroll
    for (int e = 0; e < 8; ++e) sum = __builtin_fma((double)to_f32(u.v[e]), (double)q[k + e], sum);
  }
  return group_sum_f64<LANES>(sum);
}

// Row `in` of a group.
template <int GROUP>
__device__ __forceinline__ uint64_t group_row(uint32_t group, uint32_t in) {
  return GROUP == 64 ? (uint64_t)group * 64 + in : (uint64_t)(group / 2) * 32 + in / 4 * 8 + group % 2 * 4 + in % 4;
}

// Sum over LANES (16 or 64) lanes.
template <int LANES>
__device__ __forceinline__ float lanes_sum(float v) {
  v += __int_as_float(dpp_i32<kDppQuadXor1>(__float_as_int(v)));
  v += __int_as_float(dpp_i32<kDppQuadXor2>(__float_as_int(v)));
  v += __int_as_float(dpp_i32<kDppRowHalfMirror>(__float_as_int(v)));
  v += __int_as_float(dpp_i32<kDppRowMirror>(__float_as_int(v)));
  if constexpr (LANES == 64) {
    LanePair p = lane_pair<true>(__float_as_uint(v));
    v = __uint_as_float(p.low) + __uint_as_float(p.high);
    p = lane_pair<false>(__float_as_uint(v));
    v = __uint_as_float(p.low) + __uint_as_float(p.high);
  }
  return v;
}

// One workgroup per query: joins the splits' statistics, scores the given row, finds the alternatives.  Bound by the time
// that one read after another takes, so as much as can be is read at once, and the workgroup waits for itself as seldom
// as it can.  The rows of the groups in question are scored in fp32 first, 16 lanes to a row and several rows
// of a lane in flight, and in fp64 where that leaves them among the best.
template <typename T, int GROUP, int THREADS>
__global__ __launch_bounds__(THREADS, THREADS == 256 ? 5 : 4) void row_finish_kernel(FinishArgs a) {
  constexpr int kWaves = THREADS / kWave;
  constexpr uint32_t kSharers = THREADS / kTops;  // lanes to one of the tops
  extern __shared__ __attribute__((aligned(16))) char dynamic[];
  float *q = (float *)dynamic;  // [d rounded up to 512: zeros]
  __shared__ double room64[2][kWaves];
  __shared__ float room32[4][kWaves];
  __shared__ __attribute__((aligned(16))) float tops[kTops];
  __shared__ uint32_t n_list, n_single, n_rough, n_best;
  __shared__ float kth;
  const uint32_t i = blockIdx.x, tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  const ScoreTable &g = a.g;
  const T *rows = (const T *)g.rows;
  const uint32_t n_groups = GROUP ? group_count(g.n, GROUP) : 0, stride = GROUP ? group_stride(g.n, GROUP) : 0;
  const float *gm = a.group_max + (uint64_t)i * stride;
  const uint32_t target = a.targets ? a.targets[i] : ANN_PAD_ID;
  if (tid == 0) kth = -INFINITY, n_list = 0, n_single = 0, n_rough = 0, n_best = 0;
  float qsq = 0.0f;
  for (uint32_t c = tid; c < (g.d + 511) / 512 * 512; c += THREADS) {
    const float v = c < g.d ? to_f32(((const T *)g.q)[(uint64_t)i * g.q_stride + c]) : 0.0f;
    q[c] = v;
    qsq = __builtin_fmaf(v, v, qsq);
  }
  float m = -INFINITY, x_norm = 0.0f, top = -INFINITY;
  float4 first = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  if (tid < a.splits) first = a.stats[(uint64_t)tid * g.nq + i];
  if (first.y != 0.0f) m = first.x;
  for (uint32_t s = tid + THREADS; s < a.splits; s += THREADS) {
    const float4 v = a.stats[(uint64_t)s * g.nq + i];
    if (v.y != 0.0f) m = fmaxf(m, v.x);
  }
  if constexpr (GROUP != 0) {
    for (uint32_t c = tid; c < n_groups; c += THREADS * kInFlight) {
      float v[kInFlight];
#pragma unroll
      for (uint32_t u = 0; u < kInFlight; ++u) v[u] = c + u * THREADS < n_groups ? gm[c + u * THREADS] : -INFINITY;
#pragma unroll
      for (uint32_t u = 0; u < kInFlight; ++u) top = fmaxf(top, v[u]);
    }
    for (uint32_t c = tid; c < a.norm_runs; c += THREADS) x_norm = fmaxf(x_norm, a.norms[c]);
#pragma unroll
    for (uint32_t far = 1; far < kSharers; far *= 2) top = fmaxf(top, __int_as_float(xor_lane_i32(__float_as_int(top), (int)far)));
    if (tid % kSharers == 0) tops[tid / kSharers] = top;
  }
  {
    const float wm = wave_max_f32(m), wx = wave_max_f32(x_norm), wt = wave_max_f32(top), wq = lanes_sum<64>(qsq);
    if (lane == 0) room32[0][wave] = wm, room32[1][wave] = wx, room32[2][wave] = wt, room32[3][wave] = wq;
  }
  __syncthreads();
  m = room32[0][0], x_norm = room32[1][0], qsq = room32[3][0];
  float largest = room32[2][0];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) {
    m = fmaxf(m, room32[0][w]), x_norm = fmaxf(x_norm, room32[1][w]), largest = fmaxf(largest, room32[2][w]);
    qsq += room32[3][w];
  }
  // statistics (fp64: the splits' sums are joined once)
  double l = 0.0, t = 0.0;
  const auto join_split = [&](const float4 &v) {
    if (v.y != 0.0f) {
      const double by = ((double)v.x - (double)m) * a.unit, f = exp(by);
      l += f * (double)v.y;
      t += f != 0.0 ? f * ((double)v.z * a.unit + by * (double)v.y) : 0.0;
    }
  };
  join_split(first);
  for (uint32_t s = tid + THREADS; s < a.splits; s += THREADS) join_split(a.stats[(uint64_t)s * g.nq + i]);
  l = group_sum_f64<64>(l);
  t = group_sum_f64<64>(t);
  if (lane == 0) room64[0][wave] = l, room64[1][wave] = t;
  double target_dot = 0.0;
  if (target < g.n && wave == kWaves - 1) target_dot = exact_dot<T, 64>(rows + (uint64_t)target * g.row_stride, q, g.d);
  if constexpr (GROUP != 0) {
    // The k-th largest of the tops: at least k groups reach it.
    const float own = tops[tid / kSharers];
    int above = 0;
    for (uint32_t c = tid % kSharers * (kTops / kSharers); c < (tid % kSharers + 1) * (kTops / kSharers); c += 4) {
      const float4 o = *(const float4 *)(tops + c);
      const float v[4] = {o.x, o.y, o.z, o.w};
#pragma unroll
      for (uint32_t e = 0; e < 4; ++e) above += v[e] > own || (v[e] == own && c + e < tid / kSharers);
    }
    above = group_sum_i32<(int)kSharers>(above);
    if (tid % kSharers == 0 && above == (int)a.k - 1) kth = own;
  }
  __syncthreads();
  l = room64[0][0], t = room64[1][0];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) l += room64[0][w], t += room64[1][w];
  const bool none = l == 0.0;  // no row left
  const double log_l = none ? 0.0 : log(l), shift = a.scale_error * ((double)m * a.unit + t / l);
  const double lse = none ? -INFINITY : (double)m * a.unit + log_l + (fabs(shift) < INFINITY ? shift : 0.0);
  if (wave == kWaves - 1 && lane == 0) {
    double lp = 0.0;
    if (target < g.n) {  // (an id that is no row's: none)
      const float bias = g.bias ? g.bias[target] : 0.0f;
      lp = none || bias == -INFINITY ? -INFINITY : (double)g.scale * target_dot + (double)bias - lse;
    }
    a.lse[i] = (float)lse;
    if (a.wide_lse) a.wide_lse[i] = lse;
    a.logprob[i] = lp > 0.0 ? 0.0f : (float)lp;
    const double h = none ? 0.0 : log_l - t / l;
    if (a.entropy) a.entropy[i] = h < 0.0 ? 0.0f : (float)h;
  }
  if constexpr (GROUP != 0) {
    __shared__ uint32_t list[kListed], rough[kWaves * GROUP];
    __shared__ double best[2][kBest];
    __shared__ uint32_t best_id[2][kBest];
    const float *second = GROUP == 16 && a.group_second ? a.group_second + (uint64_t)i * stride : nullptr;
    const float lost = (float)g.d * 0x1p-126f;  // squares below the smallest normal number may have gone
    const float error = score_room(g.d, sizeof(T) == 4, second != nullptr, sqrtf(qsq + lost), sqrtf(x_norm + lost), g.scale, fmaxf(fabsf(largest), fabsf(kth)));
    const bool bounded = error < INFINITY && kth > -INFINITY;  // (false with NaN)
    const float least = bounded ? kth - 2.0f * error : -INFINITY;
    double bound = bounded ? (double)kth - (double)error : -INFINITY;  // the k-th score is at least this
    uint32_t side = 0;
    // Place of candidate c among the candidates.
    const auto place = [&](uint32_t c, uint32_t count) {
      const double s = best[side][c];
      const uint32_t id = best_id[side][c];
      uint32_t rank = 0;
      for (uint32_t o = 0; o < count; ++o) rank += best[side][o] > s || (best[side][o] == s && best_id[side][o] < id);
      return rank;
    };
    const auto keep_best = [&]() {  // the k best of the candidates, in order; all lanes
      __syncthreads();
      const uint32_t count = n_best;
      for (uint32_t c = tid; c < count; c += THREADS) {
        const uint32_t rank = place(c, count);
        if (rank < a.k) best[side ^ 1][rank] = best[side][c], best_id[side ^ 1][rank] = best_id[side][c];
      }
      __syncthreads();
      side ^= 1;
      if (tid == 0) n_best = count < a.k ? count : a.k;
      if (count >= a.k && best[side][a.k - 1] > bound) bound = best[side][a.k - 1];
      __syncthreads();
    };
    constexpr uint32_t LANES = 16;  // to a row (64: a fifth slower with 768 columns, like with 128 of them)
    constexpr int kRows = THREADS == 256 || GROUP == 16 ? 4 : 8;  // of a lane in flight
    // All groups at once, or, where more are in question than the list holds, as many as it holds at a time.
    uint32_t begin = 0, end = n_groups;
    while (begin < n_groups) {
      for (uint32_t c = begin + tid; c < end; c += THREADS * kInFlight) {
        float v[kInFlight];
#pragma unroll
        for (uint32_t u = 0; u < kInFlight; ++u) v[u] = c + u * THREADS < end ? gm[c + u * THREADS] : NAN;
#pragma unroll
        for (uint32_t u = 0; u < kInFlight; ++u)
          // (the order plays no part; not bounded: every group, a NaN may have hidden its other rows)
          if (v[u] >= least || (!bounded && c + u * THREADS < end)) {
            const uint32_t group = c + u * THREADS;
            if (bounded && second && !(second[group] >= least)) {  // one row of it: from the list's end
              const uint32_t at = atomicAdd(&n_single, 1u);
              if (at < kListed) list[kListed - 1 - at] = (uint32_t)group_row<GROUP>(group, __float_as_uint(v[u]) & 15u);
            } else {
              const uint32_t at = atomicAdd(&n_list, 1u);
              if (at < kListed) list[at] = group;
            }
          }
      }
      __syncthreads();
      const uint32_t count = n_list, singles = n_single;
      __syncthreads();
      if (tid == 0) n_list = 0, n_single = 0;
      if (count + singles > kListed) {  // (of all groups)
        end = kListed;
        __syncthreads();
        continue;
      }
      // Scores rows in fp64, a wavefront to a row (short ones: 16 lanes), and keeps what may be among the best.  All lanes.
      const auto score_some = [&](auto lanes, const uint32_t *ids, int step, uint32_t found, bool first_of_all) {
        constexpr int LANES = decltype(lanes)::value;
        constexpr uint32_t kAtOnce = THREADS / LANES;
        for (uint32_t f0 = 0; f0 < found; f0 += kAtOnce) {
          if (f0 != 0 || !first_of_all) {  // (at first there is room)
            const uint32_t held = n_best;
            __syncthreads();  // all lanes have read it: they agree whether to make more
            if (held + kAtOnce > kBest) keep_best();
          }
          const uint32_t f = f0 + tid / LANES;
          if (f < found) {
            const uint32_t row = ids[(int)f * step];
            const float bias = row < g.n ? (g.bias ? g.bias[row] : 0.0f) : -INFINITY;
            const double s = bias != -INFINITY ? (double)g.scale * exact_dot<T, LANES>(rows + row * g.row_stride, q, g.d) + (double)bias : (double)NAN;
            if (lane % LANES == 0 && s >= bound) {
              const uint32_t at = atomicAdd(&n_best, 1u);
              best[side][at] = s, best_id[side][at] = row;
            }
          }
          __syncthreads();
        }
      };
      const auto score_rows = [&](const uint32_t *ids, int step, uint32_t found, bool first_of_all) {
        if (g.d <= 128)
          score_some(std::integral_constant<int, 16>(), ids, step, found, first_of_all);
        else
          score_some(std::integral_constant<int, 64>(), ids, step, found, first_of_all);
      };
      score_rows(list + kListed - 1, -1, singles, begin == 0);
      for (uint32_t c0 = 0; c0 < count; c0 += kWaves) {
        const uint32_t c = c0 + wave;
        if (c < count) {
          const uint32_t group = list[c];
          for (uint32_t in0 = 0; in0 < GROUP; in0 += kWave / LANES * kRows) {
            float dot[kRows];
#pragma unroll
            for (int r = 0; r < kRows; ++r) dot[r] = 0.0f;
            for (uint32_t k0 = 0; k0 < g.d; k0 += LANES * 8) {
              const uint32_t k = k0 + lane % LANES * 8;
              Unit<T> u[kRows];
              const T *x[kRows];
#pragma unroll
              for (int r = 0; r < kRows; ++r) {  // (rows behind the last: the last once more)
                const uint64_t row = group_row<GROUP>(group, in0 + r * (kWave / LANES) + lane / LANES);
                x[r] = rows + (row < g.n ? row : g.n - 1) * g.row_stride + k;
              }
              if (k0 + LANES * 8 <= g.d) {
#pragma unroll
                for (int r = 0; r < kRows; ++r) load_unit(u[r], x[r]);
              } else {
#pragma unroll
                for (int r = 0; r < kRows; ++r) load_unit(u[r], x[r], (int64_t)g.d - k);
              }
#pragma unroll
              for (int e = 0; e < 8; ++e) {
                const float v = q[k + e];
#pragma unroll
                for (int r = 0; r < kRows; ++r) dot[r] = __builtin_fmaf(to_f32(u[r].v[e]), v, dot[r]);
              }
            }
#pragma unroll
            for (int r = 0; r < kRows; ++r) {
              const uint64_t row = group_row<GROUP>(group, in0 + r * (kWave / LANES) + lane / LANES);
              const float bias = row < g.n ? (g.bias ? g.bias[row] : 0.0f) : -INFINITY;
              const float s = __builtin_fmaf(lanes_sum<LANES>(dot[r]), g.scale, bias);
              // (not bounded: whatever is not left out; a score that is NaN in fp64 as well is dropped there)
              if (lane % LANES == 0 && bias != -INFINITY && (!bounded || (double)s >= bound - (double)error)) rough[atomicAdd(&n_rough, 1u)] = (uint32_t)row;
            }
          }
        }
        __syncthreads();
        const uint32_t found = n_rough;
        score_rows(rough, 1, found, (begin | c0 | singles) == 0);
        if (tid == 0) n_rough = 0;
        __syncthreads();
      }
      __syncthreads();  // (the list has been read; n_list is zero)
      begin = end;
      end = end + kListed < n_groups ? end + kListed : n_groups;
    }
    const uint32_t count = n_best;
    for (uint32_t c = tid; c < count; c += THREADS) {
      const uint32_t rank = place(c, count);
      if (rank < a.k) {
        const double lp = best[side][c] - lse;
        a.alt_ids[(uint64_t)i * a.k + rank] = best_id[side][c];
        a.alt_logprobs[(uint64_t)i * a.k + rank] = lp > 0.0 ? 0.0f : (float)lp;
      }
    }
    for (uint32_t c = count + tid; c < a.k; c += THREADS) {
      a.alt_ids[(uint64_t)i * a.k + c] = ANN_PAD_ID;
      a.alt_logprobs[(uint64_t)i * a.k + c] = -INFINITY;
    }
  }
}

// ---------------------------------------------------------------------------
struct ForwardPlan {
  uint32_t q_tiles = 0, splits = 0, norm_runs = 0;
  int group = 0;
  int blocks = 0;  // of 16 queries, if the rows are streamed
  int slices = 0;  // of 16 columns, if the queries stay in registers
  bool wide = false;  // tiles of 256 rows
  uint64_t stats_at = 0, groups_at = 0, seconds_at = 0, norms_at = 0;
  bool numbered = false;
  Parts parts;
};

// Bytes of queries in LDS that the streaming kernel would take.
static uint64_t stream_lds(int blocks, uint32_t d, uint32_t type) {
  const uint64_t queries = (d + 31) / 32 * (type == ANN_F32 ? 3ull : 1ull) * blocks * 1024, stats = sizeof(Stats) * 16ull * blocks * (kStreamThreads / kWave);
  return queries > stats ? queries : stats;
}

static ForwardPlan forward_plan(uint32_t nq, uint64_t n, uint32_t d, uint32_t type, uint32_t k) {
  ForwardPlan p;
  if (nq == 0 || n == 0) return p;
  // (four blocks of fp32 queries and the rows' parts are more registers than a wavefront has)
  const int blocks = nq <= 16 ? 1 : nq <= 32 ? 2 : 4;
  if (nq <= (type == ANN_F32 ? 32 : 64) && stream_lds(blocks, d, type) <= kStreamLds) {
    p.blocks = blocks;
    const uint64_t most = (n + kStreamRows - 1) / kStreamRows;
    p.splits = most < kStreamGroups ? (uint32_t)most : kStreamGroups;
  } else {
    const bool rows_short = type != ANN_F32 && d <= 128;
    if (rows_short) p.slices = d <= 32 ? 2 : d <= 64 ? 4 : d <= 96 ? 6 : 8;
    const uint32_t queries = rows_short ? kShortQueries : kTile;
    p.q_tiles = (nq + queries - 1) / queries;
    // (tiles of 256 rows where they still fill the card)
    p.wide = !rows_short && type != ANN_F32 && d % kWideSlice == 0 && p.q_tiles * ((n + 2 * kTile - 1) / (2 * kTile)) >= kWideSlots;
    const uint32_t rows = rows_short ? kShortRows : p.wide ? 2 * kTile : kTile;
    const uint32_t row_tiles = (uint32_t)((n + rows - 1) / rows);
    uint32_t want = (kSplitTarget + p.q_tiles - 1) / p.q_tiles;
    want = (want + 7) / 8 * 8;
    if (p.wide) {
      // few rounds of workgroups whose last one is as full as can be: the least rounds times tiles
      uint64_t least = ~0ull;
      for (uint32_t s = ((kWideSlots + p.q_tiles - 1) / p.q_tiles + 7) / 8 * 8, end = s * 4; s <= end; s += 8) {
        const uint64_t cost = ((uint64_t)p.q_tiles * s + kWideSlots - 1) / kWideSlots * ((row_tiles + s - 1) / s);
        if (cost < least) least = cost, want = s;
      }
    }
    p.splits = want < row_tiles ? want : row_tiles;
  }
  // What a group costs: 8 n / group bytes per query written and read, and about k group d elements read again; of a
  // numbered one of 16 (long rows, where the end of a tile is a small part) 12 n / 16 bytes and mostly k rows.
  p.numbered = k && !p.blocks && !p.slices;
  if (p.numbered)
    p.group = n / 8 + 64ull * k * d * type_bytes(type) <= 12 * n / 16 + (uint64_t)k * d * type_bytes(type) ? 64 : 16;
  else if (k)
    p.group = 4 * n >= 1024ull * k * d ? 64 : 16;
  p.numbered = p.numbered && p.group == 16;
  p.stats_at = p.parts.take((uint64_t)p.splits * nq * sizeof(float4));
  if (k) {
    p.groups_at = p.parts.take((uint64_t)nq * group_stride((uint32_t)n, p.group) * sizeof(float));
    if (p.numbered) p.seconds_at = p.parts.take((uint64_t)nq * group_stride((uint32_t)n, 16) * sizeof(float));
    p.norm_runs = p.blocks ? p.splits : (uint32_t)((n + 15) / 16 < kNormRuns ? (n + 15) / 16 : kNormRuns);
    p.norms_at = p.parts.take(p.norm_runs * sizeof(float));
  }
  return p;
}

// Query tiles that a die takes together: as many as fill a quarter of its L2, at most eight.
static uint32_t query_group(uint32_t q_tiles, uint32_t d, uint32_t elem) {
  uint32_t group = 8;
  while (group > 1 && (group * kTile * (uint64_t)d * elem > (1u << 20) || group > q_tiles)) group /= 2;
  return group;
}
static uint32_t query_grid(uint32_t q_tiles, uint32_t group, uint32_t splits) { return ((q_tiles + group - 1) / group * splits + 7) / 8 * 8 * group; }

template <typename T>
static ann_status forward(const ann_row_scores &s, uint32_t k, const ForwardPlan &p, FinishArgs f, char *ws, hipStream_t st, bool apart = false) {
  const ScoreTable &g = f.g;
  if (s.n) {
    float4 *stats = (float4 *)(ws + p.stats_at);
    float *groups = (float *)(ws + p.groups_at), *seconds = p.numbered ? (float *)(ws + p.seconds_at) : nullptr, *norms = (float *)(ws + p.norms_at);
    const bool bias = g.bias || g.scale < 0.0f;
    hipError_t refused = hipSuccess;
    const auto run = [&](auto with_bias, auto group) {
      constexpr bool BIAS = decltype(with_bias)::value;
      constexpr int GROUP = decltype(group)::value;
      if (!p.blocks) {
        // (rows too far apart for the offsets of the kernel for short ones: the other one, with as many splits)
        const bool is_short = p.slices && g.row_stride <= kShortStride;
        const uint32_t q_tiles = is_short ? p.q_tiles : (g.nq + kTile - 1) / kTile, grid = q_tiles * ((p.splits + 7) / 8 * 8);
        const auto rows_short = [&](auto slices) {
          if constexpr (sizeof(T) == 2) row_scores_short_kernel<T, decltype(slices)::value, BIAS, GROUP><<<grid, 256, 0, st>>>(g, q_tiles, p.splits, stats, groups);
        };
        const uint32_t q_group = query_group(q_tiles, g.d, sizeof(T)), paired = query_grid(q_tiles, q_group, p.splits);
        if (p.wide && wide_operand(g.q, g.q_stride) && wide_operand(g.rows, g.row_stride)) {
          if constexpr (sizeof(T) == 2) row_scores_kernel<T, BIAS, GROUP, 4><<<paired, 256, 0, st>>>(g, q_tiles, q_group, p.splits, stats, groups, seconds);
        } else if (!is_short && apart) {
          if constexpr (sizeof(T) == 4 && GROUP == 0) row_scores_kernel<T, BIAS, GROUP, 2, true><<<paired, 256, 0, st>>>(g, q_tiles, q_group, p.splits, stats, groups, seconds);
        } else if (!is_short)
          row_scores_kernel<T, BIAS, GROUP, 2><<<paired, 256, 0, st>>>(g, q_tiles, q_group, p.splits, stats, groups, seconds);
        else if (p.slices == 2)
          rows_short(std::integral_constant<int, 2>());
        else if (p.slices == 4)
          rows_short(std::integral_constant<int, 4>());
        else if (p.slices == 6)
          rows_short(std::integral_constant<int, 6>());
        else
          rows_short(std::integral_constant<int, 8>());
        if (GROUP) row_norms_kernel<T><<<p.norm_runs, 256, 0, st>>>(g, norms);
        return;
      }
      const auto stream = [&](auto blocks) {
        const auto kernel = row_stream_kernel<T, decltype(blocks)::value, BIAS, GROUP>;
        const uint32_t lds = (uint32_t)stream_lds(p.blocks, g.d, s.type);
        if (lds > 64u << 10) refused = hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (refused == hipSuccess) kernel<<<p.splits, kStreamThreads, lds, st>>>(g, stats, groups, norms);
      };
      if (p.blocks == 1)
        stream(std::integral_constant<int, 1>());
      else if (p.blocks == 2)
        stream(std::integral_constant<int, 2>());
      else if constexpr (sizeof(T) == 2)
        stream(std::integral_constant<int, 4>());
    };
    const auto run_group = [&](auto with_bias) {
      if (p.group == 0)
        run(with_bias, std::integral_constant<int, 0>());
      else if (p.group == 16)
        run(with_bias, std::integral_constant<int, 16>());
      else
        run(with_bias, std::integral_constant<int, 64>());
    };
    if (bias)
      run_group(std::true_type());
    else
      run_group(std::false_type());
    ANN_HIP(refused);
    ANN_HIP(hipGetLastError());
    f.stats = stats, f.group_max = groups, f.group_second = seconds, f.norms = norms, f.splits = p.splits, f.norm_runs = p.norm_runs;
    const float c = g.scale * kLog2e;
    f.unit = bias ? 1.0 : M_LN2;
    f.scale_error = bias || c == 0.0f ? 0.0 : (double)g.scale * M_LOG2E / (double)c - 1.0;
  }
  const uint32_t lds = (g.d + 511) / 512 * 512 * sizeof(float);
  const auto end = [&](auto group) {
    constexpr int GROUP = decltype(group)::value;
    // (few queries: what one of them takes counts, and 16 wavefronts read its groups at once)
    if (s.nq < kFewQueries)
      row_finish_kernel<T, GROUP, 1024><<<s.nq, 1024, lds, st>>>(f);
    else
      row_finish_kernel<T, GROUP, 256><<<s.nq, 256, lds, st>>>(f);
  };
  if (k == 0)
    end(std::integral_constant<int, 0>());
  else if (p.group == 16)
    end(std::integral_constant<int, 16>());
  else
    end(std::integral_constant<int, 64>());
  ANN_HIP(hipGetLastError());
  return ANN_OK;
}

ann_status row_statistics(const ann_row_scores &s, float *logprob, float *lse, double *wide_lse, void *workspace, hipStream_t st) {
  const ForwardPlan p = forward_plan(s.nq, s.n, s.d, s.type, 0);
  FinishArgs f = {};
  f.g = score_table(s), f.logprob = logprob, f.lse = lse, f.wide_lse = wide_lse;
  if (s.type == ANN_F32) return forward<float>(s, 0, p, f, (char *)workspace, st, true);
  if (s.type == ANN_F16) return forward<f16_t>(s, 0, p, f, (char *)workspace, st);
  return forward<bf16_t>(s, 0, p, f, (char *)workspace, st);
}

ann_status check_scores(const char *what, const ann_row_scores *s) {
  if (!s) return fail(ANN_EINVAL, "%s: scores is NULL", what);
  if (s->type > ANN_BF16) return fail(ANN_EINVAL, "%s: unknown type %u", what, s->type);
  if (s->d == 0) return fail(ANN_EINVAL, "%s: d == 0", what);
  if (s->d > ANN_MAX_SCORE_DIM) return fail(ANN_ECAPACITY, "%s: d = %u exceeds ANN_MAX_SCORE_DIM = %u", what, s->d, ANN_MAX_SCORE_DIM);
  if (s->n > kMaxRows || s->nq >= kMaxQueries) return fail(ANN_ECAPACITY, "%s: n must be at most 2^31 - 256 and nq below 2^24", what);
  if (!(fabsf(s->scale) < INFINITY)) return fail(ANN_EINVAL, "%s: scale must be finite", what);
  if (s->nq && (!s->q || s->q_stride < s->d)) return fail(ANN_EINVAL, "%s: q is NULL or its stride shorter than a row", what);
  if (s->n && (!s->rows || s->row_stride < s->d)) return fail(ANN_EINVAL, "%s: rows is NULL or its stride shorter than a row", what);
  return ANN_OK;
}

ann_status check_workspace(const char *what, const void *workspace, uint64_t bytes, uint64_t need) {
  if (need && !workspace) return fail(ANN_EINVAL, "%s: workspace is NULL", what);
  if (bytes < need)
    return fail(ANN_EINVAL, "%s: workspace of %llu bytes, %llu are needed", what, (unsigned long long)bytes, (unsigned long long)need);
  if (need && (uintptr_t)workspace % 16) return fail(ANN_EINVAL, "%s: workspace is not aligned to 16 bytes", what);
  return ANN_OK;
}

}  // namespace ann

using namespace ann;

extern "C" uint64_t ann_row_logprobs_workspace(uint32_t nq, uint64_t n, uint32_t d, uint32_t type, uint32_t k) {
  if (n > kMaxRows || nq >= kMaxQueries || k > ANN_MAX_ALTERNATIVES) return 0;
  return forward_plan(nq, n, d, type, k).parts.bytes;
}

extern "C" ann_status ann_row_logprobs(const ann_row_scores *scores, uint32_t k, float *logprob, float *entropy, float *lse, uint32_t *alt_ids,
                                       float *alt_logprobs, void *workspace, uint64_t workspace_bytes, void *stream) {
  if (ann_status s = check_scores("ann_row_logprobs", scores)) return s;
  if (k > ANN_MAX_ALTERNATIVES) return fail(ANN_ECAPACITY, "ann_row_logprobs: k = %u exceeds ANN_MAX_ALTERNATIVES = %u", k, ANN_MAX_ALTERNATIVES);
  if (scores->nq == 0) return ANN_OK;
  if (!logprob || !lse) return fail(ANN_EINVAL, "ann_row_logprobs: logprob or lse is NULL");
  if ((k != 0) != (alt_ids != nullptr) || (k != 0) != (alt_logprobs != nullptr))
    return fail(ANN_EINVAL, "ann_row_logprobs: alt_ids and alt_logprobs go with k > 0, k = %u", k);
  const ForwardPlan p = forward_plan(scores->nq, scores->n, scores->d, scores->type, k);
  if (ann_status s = check_workspace("ann_row_logprobs", workspace, workspace_bytes, p.parts.bytes)) return s;
  FinishArgs f = {};
  f.g = score_table(*scores);
  f.targets = scores->targets, f.k = k;
  f.logprob = logprob, f.entropy = entropy, f.lse = lse, f.alt_ids = alt_ids, f.alt_logprobs = alt_logprobs;
  if (scores->type == ANN_F32) return forward<float>(*scores, k, p, f, (char *)workspace, (hipStream_t)stream);
  if (scores->type == ANN_F16) return forward<f16_t>(*scores, k, p, f, (char *)workspace, (hipStream_t)stream);
  return forward<bf16_t>(*scores, k, p, f, (char *)workspace, (hipStream_t)stream);
}
