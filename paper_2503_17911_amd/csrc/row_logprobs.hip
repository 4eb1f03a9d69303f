// Log probabilities of given rows under the softmax of all rows' scores
// s[i][j] = scale <q_i, x_j> + bias_j, with the softmax' entropy and its largest
// alternatives.  The scores stay in the accumulators of the product: each lane
// keeps, for its queries, a running maximum m, l = sum exp(s - m) and
// t = sum exp(s - m) (s - m) (all fp32) over the rows that pass by; at the end
// lse = m + log l, entropy = log l - t / l.
//
// Alternatives: the product kernel also writes the largest score of every group of
// rows (one number for kGroup scores).  The k best rows lie in groups whose
// largest score is at least the k-th largest of those; a score may err by what
// score_room() allows, so groups within twice that below it are taken as well,
// and their rows are scored again in fp64 and put in order.  That is exact whatever the
// distribution, ties included; how many rows are scored again is all that depends on it.
#include "row_logprobs.hpp"

#include <math.h>

namespace ann {

constexpr uint32_t kNormRuns = 512;     // workgroups that look for the largest row norm
constexpr uint32_t kSplitTarget = 1536; // workgroups of the product kernel: two rounds of three to a compute unit
constexpr float kNothing = -1000.0f;    // an exponent whose power is zero, and finite

struct Stats {
  float m, l, t;
};
__device__ __forceinline__ void join(Stats &a, const Stats &b) {
  const float m = fmaxf(a.m, b.m);
  const float da = fmaxf(a.m - m, kNothing), db = fmaxf(b.m - m, kNothing);
  const float fa = __builtin_amdgcn_exp2f(da * kLog2e), fb = __builtin_amdgcn_exp2f(db * kLog2e);
  a.t = fa * __builtin_fmaf(da, a.l, a.t) + fb * __builtin_fmaf(db, b.l, b.t);
  a.l = __builtin_fmaf(fa, a.l, fb * b.l);
  a.m = m;
}

// A lane's running statistics of one query.  The scores of a tile are summed by themselves and the tiles' sums
// with what the last addition lost: over a million rows plain sums erred by 4.6e-6, ten times the rounding of the scores.
struct Running {
  float m = -3.402823466e38f, l = 0.0f, t = 0.0f, l_lost = 0.0f, t_lost = 0.0f;

  static __device__ __forceinline__ void add(float &sum, float &lost, float v) {
    v -= lost;
    const float next = sum + v;
    lost = (next - sum) - v;
    sum = next;
  }
  // N scores and the largest of them.  MASKED: they are whole, and -infinity means a row left out; otherwise a score
  // is s * scale, with c = scale log2 e.
  template <bool MASKED, int N>
  __device__ __forceinline__ void take(const float (&s)[N], float top, float c) {
    const float next = fmaxf(m, top), step = fmaxf(m - next, kNothing), f = __builtin_amdgcn_exp2f(step * kLog2e);
    // (for the same maximum: f = 1, step = 0, and these change nothing)
    t = f * __builtin_fmaf(step, l, t), t_lost *= f;
    l *= f, l_lost *= f;
    m = next;
    float sum = 0.0f, weighed = 0.0f;
    const float m2 = m * kLog2e;
#pragma unroll
    for (int r = 0; r < N; ++r) {
      if constexpr (MASKED) {
        const float y = s[r] == -INFINITY ? kNothing : s[r] - m;
        const float p = __builtin_amdgcn_exp2f(y * kLog2e);
        sum += p;
        weighed = __builtin_fmaf(p, y, weighed);
      } else {
        const float y = __builtin_fmaf(s[r], c, -m2);
        const float p = __builtin_amdgcn_exp2f(y);
        sum += p;
        weighed = __builtin_fmaf(p, y, weighed);
      }
    }
    add(l, l_lost, sum);
    add(t, t_lost, MASKED ? weighed : weighed * kLn2);
  }
  __device__ __forceinline__ Stats stats() const { return {m, l, t}; }
};

// Rows of a group of 64: a wavefront's of a tile.  Of a group of 16: those of one half of the lanes in a block of 32.
__host__ __device__ constexpr uint32_t group_count(uint32_t n, int group) { return group == 64 ? (n + 63) / 64 : (n + 31) / 32 * 2; }

// BIAS: rows may be left out, or the scale is negative.
template <typename T, bool BIAS, int GROUP>
__global__ __launch_bounds__(256) void row_scores_kernel(ScoreTable g, uint32_t q_tiles, uint32_t splits, float4 *__restrict__ stats,
                                                         float *__restrict__ group_max) {
  __shared__ __attribute__((aligned(16))) char lds[kTileBytes<T, kAlong, kAlong>];
  __shared__ float row_bias[kTile];
  // workgroup b runs on die b mod 8: a die takes all queries through its own part of the rows
  const uint32_t b8 = blockIdx.x / 8, qt = b8 % q_tiles, split = b8 / q_tiles * 8 + blockIdx.x % 8;
  if (split >= splits) return;
  const uint32_t row_tiles = (g.n + kTile - 1) / kTile;
  const uint32_t first = (uint32_t)((uint64_t)row_tiles * split / splits), last = (uint32_t)((uint64_t)row_tiles * (split + 1) / splits);
  const int wave = (int)threadIdx.x / kWave, lane = lane_id(), mw = wave / 2 * 64, nw = wave % 2 * 64;
  const Lines<T> X = {(const T *)g.rows, g.row_stride, g.n, g.d}, Q = {(const T *)g.q, g.q_stride, g.nq, g.d};
  const uint32_t n_groups = GROUP ? group_count(g.n, GROUP) : 0;
  const float c = g.scale * kLog2e;
  Running run[2];
  for (uint32_t tile = first; tile < last; ++tile) {
    const uint32_t row0 = tile * kTile;
    const bool whole = row0 + kTile <= g.n;
    f32x16 acc[2][2];
    clear(acc);
    tile_product<T, kAlong, kAlong>(acc, X, row0, Q, qt * kTile, 0, g.d, lds);
    if (BIAS || !whole) {
      // (read by the tile before's epilogue: the barriers of the product lie in between; d > 0)
      if (threadIdx.x < kTile) row_bias[threadIdx.x] = row0 + threadIdx.x < g.n ? (BIAS && g.bias ? g.bias[row0 + threadIdx.x] : 0.0f) : -INFINITY;
      __syncthreads();
    }
    const auto finish = [&](auto masked) {
      constexpr bool MASKED = decltype(masked)::value;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        float top[2];
        if constexpr (MASKED) {
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
              const float bias = row_bias[mw + i * 32 + block_row(r)];
              acc[i][j][r] = bias == -INFINITY ? -INFINITY : __builtin_fmaf(acc[i][j][r], g.scale, bias);
            }
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          top[i] = acc[i][j][0];
#pragma unroll
          for (int r = 1; r < 16; ++r) top[i] = fmaxf(top[i], acc[i][j][r]);
          if constexpr (!MASKED) top[i] *= g.scale;
        }
        if constexpr (GROUP != 0) {
          const uint32_t q = qt * kTile + nw + j * 32 + lane % 32;
          if constexpr (GROUP == 64) {
            const float both = fmaxf(top[0], top[1]);
            const LanePair p = lane_pair<false>(__float_as_uint(both));
            const float all = fmaxf(__uint_as_float(p.low), __uint_as_float(p.high));
            const uint32_t at = (row0 + mw) / 64;
            if (lane < 32 && q < g.nq && at < n_groups) group_max[(uint64_t)q * n_groups + at] = all;
          } else {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const uint32_t at = (row0 + mw + i * 32) / 32 * 2 + lane / 32;
              if (q < g.nq && at < n_groups) group_max[(uint64_t)q * n_groups + at] = top[i];
            }
          }
        }
        float all[32];
#pragma unroll
        for (int r = 0; r < 32; ++r) all[r] = acc[r / 16][j][r % 16];
        run[j].template take<MASKED>(all, fmaxf(top[0], top[1]), c);
      }
    };
    if (BIAS || !whole)
      finish(std::true_type());
    else
      finish(std::false_type());
  }
  // the two halves of a wavefront, then the two wavefronts that share queries
  __shared__ Stats other[2][64];
  Stats st[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    st[j] = run[j].stats();
    const LanePair m = lane_pair<false>(__float_as_uint(st[j].m)), l = lane_pair<false>(__float_as_uint(st[j].l)), t = lane_pair<false>(__float_as_uint(st[j].t));
    Stats a = {__uint_as_float(m.low), __uint_as_float(l.low), __uint_as_float(t.low)};
    const Stats b = {__uint_as_float(m.high), __uint_as_float(l.high), __uint_as_float(t.high)};
    join(a, b);
    st[j] = a;
    if (wave >= 2 && lane < 32) other[wave % 2][j * 32 + lane] = a;
  }
  __syncthreads();
  if (wave < 2 && lane < 32) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      join(st[j], other[wave][j * 32 + lane]);
      const uint32_t q = qt * kTile + nw + j * 32 + lane;
      if (q < g.nq) stats[(uint64_t)split * g.nq + q] = make_float4(st[j].m, st[j].l, st[j].t, 0.0f);
    }
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
  const uint32_t n_groups = GROUP ? group_count(g.n, GROUP) : 0;
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
  Running run[NB];
  f32x4 acc[NB][4];
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
        for (int b = 0; b < 4; ++b) acc[j][b] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
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
            for (int j = 0; j < NB; ++j) acc[j][b] = small_step(x[p], q[sum - p][j], acc[j][b]);
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
              s[i] = acc[j][b][r];
              if constexpr (MASKED) s[i] = bias[i] == -INFINITY ? -INFINITY : __builtin_fmaf(s[i], g.scale, bias[i]);
              top[b] = r ? fmaxf(top[b], s[i]) : s[i];
            }
            if constexpr (!MASKED) top[b] *= g.scale;
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
            float *out = group_max + (uint64_t)q * n_groups;
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
          run[j].template take<MASKED>(s, all, c);
        }
      };
      if (BIAS || !whole)
        finish(std::true_type());
      else
        finish(std::false_type());
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
      join(a, b);
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
    for (int w = 1; w < kWaves; ++w) join(a, room[w * NB * 16 + threadIdx.x]);
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
// product and addition round a score.  fp32: six products to an element.
__device__ __forceinline__ float score_room(uint32_t d, bool parts, float q_norm, float x_norm, float scale, float largest) {
  const float size = fabsf(scale) * q_norm * x_norm * 1.001f;
  return ((parts ? 6.0f : 1.0f) * (float)d + 64.0f) * 0x1p-23f * size + 0x1p-22f * (fabsf(largest) + size);
}

constexpr int kFinishThreads = 256;
constexpr uint32_t kGroupRange = 4096;  // groups that are looked through at a time
constexpr uint32_t kBest = 1024;        // candidates that are kept at a time

struct FinishArgs {
  ScoreTable g;
  const uint32_t *targets;
  const float4 *stats;
  const float *group_max, *norms;
  uint32_t splits, k, norm_runs;
  float *logprob, *entropy, *lse, *alt_logprobs;
  uint32_t *alt_ids;
};

template <typename F>
__device__ __forceinline__ double block_sum(double v, double *room, F wave_index) {
  v = group_sum_f64<64>(v);
  __syncthreads();
  if (lane_id() == 0) room[wave_index] = v;
  __syncthreads();
  double s = 0.0;
#pragma unroll
  for (int w = 0; w < kFinishThreads / kWave; ++w) s += room[w];
  return s;
}
__device__ __forceinline__ float block_max(float v, float *room) {
  v = wave_max_f32(v);
  __syncthreads();
  if (lane_id() == 0) room[threadIdx.x / kWave] = v;
  __syncthreads();
  float s = room[0];
#pragma unroll
  for (int w = 1; w < kFinishThreads / kWave; ++w) s = fmaxf(s, room[w]);
  return s;
}

// The part of lane `part` of LPR of a row's product with the query (in LDS), in fp64.
template <typename T, int LPR>
__device__ __forceinline__ double exact_dot(const T *x, const float *q, uint32_t d, uint32_t part) {
  double sum = 0.0;
  for (uint32_t k = part * 8; k < d; k += LPR * 8) {
    Unit<T> u;
    load_unit(u, x + k, (int64_t)d - k);
#pragma unroll
    for (int e = 0; e < 8; ++e) sum = __builtin_fma((double)to_f32(u.v[e]), (double)q[k + e], sum);  // (q is zero from d on)
  }
  return sum;
}

// One workgroup per query: joins the splits' statistics, scores the given row, finds the alternatives.
template <typename T, int GROUP>
__global__ __launch_bounds__(kFinishThreads) void row_finish_kernel(FinishArgs a) {
  extern __shared__ __attribute__((aligned(16))) char dynamic[];
  float *q = (float *)dynamic;  // [d rounded up to 8]
  __shared__ double room[kFinishThreads / kWave];
  __shared__ float room32[kFinishThreads / kWave];
  const uint32_t i = blockIdx.x, tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  const ScoreTable &g = a.g;
  const uint32_t d8 = (g.d + 7) / 8 * 8;
  float qsq = 0.0f;
  for (uint32_t c = tid; c < d8; c += kFinishThreads) {
    const float v = c < g.d ? to_f32(((const T *)g.q)[(uint64_t)i * g.q_stride + c]) : 0.0f;
    q[c] = v;
    qsq = __builtin_fmaf(v, v, qsq);
  }
  // statistics (fp64: the splits' sums are joined once)
  float m = -INFINITY;
  for (uint32_t s = tid; s < a.splits; s += kFinishThreads) {
    const float4 v = a.stats[(uint64_t)s * g.nq + i];
    if (v.y != 0.0f) m = fmaxf(m, v.x);
  }
  m = block_max(m, room32);
  double l = 0.0, t = 0.0;
  for (uint32_t s = tid; s < a.splits; s += kFinishThreads) {
    const float4 v = a.stats[(uint64_t)s * g.nq + i];
    if (v.y != 0.0f) {
      const double by = (double)v.x - (double)m, f = exp(by);
      l += f * (double)v.y;
      t += f != 0.0 ? f * ((double)v.z + by * (double)v.y) : 0.0;
    }
  }
  l = block_sum(l, room, wave);
  t = block_sum(t, room, wave);
  const bool none = l == 0.0;  // no row left
  const double log_l = none ? 0.0 : log(l), lse = none ? -INFINITY : (double)m + log_l;
  double target_dot = 0.0;
  const uint32_t target = a.targets ? a.targets[i] : ANN_PAD_ID;
  const bool given = target < g.n;  // (an id that is no row's: none)
  if (given && wave == 0) target_dot = group_sum_f64<64>(exact_dot<T, 64>((const T *)g.rows + (uint64_t)target * g.row_stride, q, g.d, lane));
  if (tid == 0) {
    a.lse[i] = (float)lse;
    if (a.entropy) {
      const double h = none ? 0.0 : log_l - t / l;
      a.entropy[i] = h < 0.0 ? 0.0f : (float)h;
    }
    double lp = 0.0;
    if (given) {
      const float bias = g.bias ? g.bias[target] : 0.0f;
      lp = none || bias == -INFINITY ? -INFINITY : (double)g.scale * target_dot + (double)bias - lse;
    }
    a.logprob[i] = lp > 0.0 ? 0.0f : (float)lp;
  }
  if constexpr (GROUP != 0) {
    __shared__ float tops[kFinishThreads];
    __shared__ uint32_t list[kGroupRange], n_list, n_best;
    __shared__ double best[2][kBest];
    __shared__ uint32_t best_id[2][kBest];
    __shared__ float kth;
    const uint32_t n_groups = group_count(g.n, GROUP);
    const float *gm = a.group_max + (uint64_t)i * n_groups;
    float x_norm = 0.0f, top = -INFINITY;
    for (uint32_t c = tid; c < a.norm_runs; c += kFinishThreads) x_norm = fmaxf(x_norm, a.norms[c]);
    const float lost = (float)g.d * 0x1p-126f;  // squares below the smallest normal number may have gone
    x_norm = sqrtf(block_max(x_norm, room32) + lost);
    const float q_norm = sqrtf((float)block_sum((double)qsq, room, wave) + lost);
    for (uint32_t c = tid; c < n_groups; c += kFinishThreads) top = fmaxf(top, gm[c]);
    // The k-th largest of the lanes' maxima: at least k groups reach it.
    tops[tid] = top;
    if (tid == 0) kth = -INFINITY, n_best = 0;
    __syncthreads();
    uint32_t above = 0;
    for (uint32_t c = 0; c < kFinishThreads; ++c) above += tops[c] > top || (tops[c] == top && c < tid);
    if (above == a.k - 1) kth = top;
    __syncthreads();
    const float error = score_room(g.d, sizeof(T) == 4, q_norm, x_norm, g.scale, block_max(top, room32));
    const float least = error < INFINITY ? kth - 2.0f * error : -INFINITY;  // (NaN compares false)
    double bound = (double)(kth - error < INFINITY && error < INFINITY ? kth - error : -INFINITY);  // the k-th score is at least this
    uint32_t side = 0;
    const auto keep_best = [&]() {  // the k best of the candidates, in order; all lanes
      __syncthreads();
      const uint32_t count = n_best;
      for (uint32_t c = tid; c < count; c += kFinishThreads) {
        const double s = best[side][c];
        const uint32_t id = best_id[side][c];
        uint32_t rank = 0;
        for (uint32_t o = 0; o < count; ++o) rank += best[side][o] > s || (best[side][o] == s && best_id[side][o] < id);
        if (rank < a.k) best[side ^ 1][rank] = s, best_id[side ^ 1][rank] = id;
      }
      __syncthreads();
      side ^= 1;
      if (tid == 0) n_best = count < a.k ? count : a.k;
      if (count >= a.k && best[side][a.k - 1] > bound) bound = best[side][a.k - 1];
      __syncthreads();
    };
    constexpr int kLanes = 64 / GROUP;  // to a row
    for (uint32_t begin = 0; begin < n_groups; begin += kGroupRange) {
      __syncthreads();
      if (tid == 0) n_list = 0;
      __syncthreads();
      for (uint32_t c = begin + tid; c < n_groups && c < begin + kGroupRange; c += kFinishThreads)
        if (gm[c] >= least) list[atomicAdd(&n_list, 1u)] = c;  // (the order plays no part)
      __syncthreads();
      const uint32_t count = n_list;
      for (uint32_t c0 = 0; c0 < count; c0 += kFinishThreads / kWave) {
        const uint32_t held = n_best;
        __syncthreads();  // all lanes have read it: they agree whether to make room
        if (held + kFinishThreads / kLanes > kBest) keep_best();
        const uint32_t c = c0 + wave;
        if (c < count) {
          const uint32_t group = list[c], in = lane / kLanes;
          const uint64_t row = GROUP == 64 ? (uint64_t)group * 64 + in : (uint64_t)(group / 2) * 32 + in / 4 * 8 + group % 2 * 4 + in % 4;
          const float bias = row < g.n ? (g.bias ? g.bias[row] : 0.0f) : -INFINITY;
          if (bias != -INFINITY) {
            double s = exact_dot<T, kLanes>((const T *)g.rows + row * g.row_stride, q, g.d, lane % kLanes);
            s = group_sum_f64<kLanes>(s);
            s = (double)g.scale * s + (double)bias;
            if (lane % kLanes == 0 && s >= bound) {
              const uint32_t at = atomicAdd(&n_best, 1u);
              best[side][at] = s, best_id[side][at] = (uint32_t)row;
            }
          }
        }
        __syncthreads();
      }
    }
    keep_best();
    for (uint32_t c = tid; c < a.k; c += kFinishThreads) {
      const bool is = c < n_best;
      const double lp = is ? best[side][c] - lse : -INFINITY;
      a.alt_ids[(uint64_t)i * a.k + c] = is ? best_id[side][c] : ANN_PAD_ID;
      a.alt_logprobs[(uint64_t)i * a.k + c] = lp > 0.0 ? 0.0f : (float)lp;
    }
  }
}

// ---------------------------------------------------------------------------
struct ForwardPlan {
  uint32_t q_tiles = 0, splits = 0, norm_runs = 0;
  int group = 0;
  int blocks = 0;  // of 16 queries, if the rows are streamed
  uint64_t stats_at = 0, groups_at = 0, norms_at = 0;
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
    p.q_tiles = (nq + kTile - 1) / kTile;
    const uint32_t row_tiles = (uint32_t)((n + kTile - 1) / kTile);
    uint32_t want = (kSplitTarget + p.q_tiles - 1) / p.q_tiles;
    want = (want + 7) / 8 * 8;
    p.splits = want < row_tiles ? want : row_tiles;
  }
  // What a group costs: 8 n / group bytes per query written and read, and about k group d elements read again.
  if (k) p.group = 4 * n >= 1024ull * k * d ? 64 : 16;
  p.stats_at = p.parts.take((uint64_t)p.splits * nq * sizeof(float4));
  if (k) {
    p.groups_at = p.parts.take((uint64_t)nq * group_count((uint32_t)n, p.group) * sizeof(float));
    p.norm_runs = p.blocks ? p.splits : (uint32_t)((n + 15) / 16 < kNormRuns ? (n + 15) / 16 : kNormRuns);
    p.norms_at = p.parts.take(p.norm_runs * sizeof(float));
  }
  return p;
}

template <typename T>
static ann_status forward(const ann_row_scores &s, uint32_t k, const ForwardPlan &p, FinishArgs f, char *ws, hipStream_t st) {
  const ScoreTable &g = f.g;
  if (s.n) {
    float4 *stats = (float4 *)(ws + p.stats_at);
    float *groups = (float *)(ws + p.groups_at), *norms = (float *)(ws + p.norms_at);
    const bool bias = g.bias || g.scale < 0.0f;
    hipError_t refused = hipSuccess;
    const auto run = [&](auto with_bias, auto group) {
      constexpr bool BIAS = decltype(with_bias)::value;
      constexpr int GROUP = decltype(group)::value;
      if (!p.blocks) {
        row_scores_kernel<T, BIAS, GROUP><<<p.q_tiles * ((p.splits + 7) / 8 * 8), 256, 0, st>>>(g, p.q_tiles, p.splits, stats, groups);
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
    f.stats = stats, f.group_max = groups, f.norms = norms, f.splits = p.splits, f.norm_runs = p.norm_runs;
  }
  const uint32_t lds = (g.d + 7) / 8 * 8 * sizeof(float);
  if (k == 0)
    row_finish_kernel<T, 0><<<s.nq, kFinishThreads, lds, st>>>(f);
  else if (p.group == 16)
    row_finish_kernel<T, 16><<<s.nq, kFinishThreads, lds, st>>>(f);
  else
    row_finish_kernel<T, 64><<<s.nq, kFinishThreads, lds, st>>>(f);
  ANN_HIP(hipGetLastError());
  return ANN_OK;
}

ann_status check_scores(const char *what, const ann_row_scores *s) {
  if (!s) return fail(ANN_EINVAL, "%s: scores is NULL", what);
  if (s->type > ANN_BF16) return fail(ANN_EINVAL, "%s: unknown type %u", what, s->type);
  if (s->d == 0) return fail(ANN_EINVAL, "%s: d == 0", what);
  if (s->d > ANN_MAX_SCORE_DIM) return fail(ANN_ECAPACITY, "%s: d = %u exceeds ANN_MAX_SCORE_DIM = %u", what, s->d, ANN_MAX_SCORE_DIM);
  if (s->n >= (1ull << 31) || s->nq >= (1u << 31)) return fail(ANN_ECAPACITY, "%s: n and nq must be below 2^31", what);
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
  if (n >= (1ull << 31) || nq >= (1u << 31) || k > ANN_MAX_ALTERNATIVES) return 0;
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
