// Root-mean-square norm of the rows of a matrix, with the residual's addition before it, and its gradients.
//
//   h = x + residual, rounded to the rows' type and kept;  y = h * rstd * w,  rstd = 1 / sqrt(mean(h^2) + eps)
//   dx = rstd * (a - xh * mean(a * xh)) + dsum,  a = dy * w,  xh = h * rstd;   dw = sum over rows of dy * xh
//
// The norm is that of h as it is kept, so that the gradient, which reads h again, is that of the values returned.
// In 8 bits (e4m3): v = h * rstd * w in fp32, scale = max |v| / 448 over a group of columns (or the row), code = fp32's quotient v / scale, rounded to 8 bits.
//
// Bound by memory: every row is read once and stays in the registers of 16 to 512 lanes as the pieces that were loaded (of 16 bytes with any
// alignment: rows of odd strides are read as wide as the others), one to four to a lane; sums are fp32.  A group of columns that
// shares a scale is 4 to 32 lanes side by side: its maximum takes two to five lane exchanges.  Gradients of the weights collect in registers, one
// part per workgroup, added in a fixed order by a second kernel.  Measured: 80,000 x 768 bf16 with the residual in e4m3 84 us (5.1 TB/s, as a large copy
// reaches; 83 with a multiplication in the place of the codes' division), the gradient 99 us (5.0 TB/s, of which 4.8 are the second kernel; 226 us by 64 lanes of four pieces, a third of them idle, with elements instead of
// words in registers); rows of 769: 115 us in bf16, gradient 180; one row 3 us.
#include "row_pieces.hpp"

#include <type_traits>

namespace ann {

constexpr uint32_t kRmsBlocks = 2048;   // workgroups of a pass over rows at most
constexpr uint32_t kRmsParts = 512;     // partial sums of the weights' gradient at most
constexpr float kE4m3Max = 448.0f;
constexpr float kSmallestMax = 0x1p-100f;  // of a group, as its scale takes it: the scale and its inverse stay normal numbers

struct RmsArgs {
  const void *x, *residual, *weight, *dy;  // backward: x is h, residual dsum
  void *sum, *y;                           // backward: y is dx
  float *rstd, *scales, *partial;          // partial: [workgroups][dim]
  uint64_t n, x_stride, residual_stride, sum_stride, y_stride, scale_stride, dy_stride;
  uint32_t dim, group;
  float eps;
  bool weight_f32;
};

template <int LANES>
constexpr int kRmsThreads = LANES > 256 ? LANES : 256;

// The codes of v / scale, of the VEC values from column c on: 448 is the largest that there is, v / scale is not above it but for its rounding.
// (A division: times 1 / scale, which is rounded itself, values halfway between two codes leave their place: 175 of a scale of 7.)
template <int VEC>
__device__ __forceinline__ void store_codes(const float (&v)[VEC], float scale, uint8_t *row, uint32_t c, uint32_t columns) {
  Words<VEC / 4, 1> o;
#pragma unroll
  for (int w = 0; w < VEC / 4; ++w) {
    const int low = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * w] / scale, v[4 * w + 1] / scale, 0, false);
    o.v[w] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v[4 * w + 2] / scale, v[4 * w + 3] / scale, low, true);
  }
  if (c + VEC <= columns) {
    *(Words<VEC / 4, 1> *)(row + c) = o;
  } else {
#pragma unroll
    for (int e = 0; e < VEC; ++e)
      if (c + e < columns) row[c + e] = (uint8_t)(o.v[e / 4] >> (e % 4 * 8));
  }
}

// The weights of VEC columns from c on; whatever, behind the last column.
template <typename T, int VEC, RowEnd END>
__device__ __forceinline__ void load_weights(float (&w)[VEC], const RmsArgs &g, uint32_t c) {
  if (!g.weight) {
#pragma unroll
    for (int e = 0; e < VEC; ++e) w[e] = 1.0f;
  } else if (g.weight_f32) {
#pragma unroll
    for (int p = 0; p < VEC; p += 4) {
      RowPiece<float, 4, END> piece;
      piece.load((const float *)g.weight, c + p, g.dim);
#pragma unroll
      for (int e = 0; e < 4; ++e) w[p + e] = piece.get(e);
    }
  } else {
    RowPiece<T, VEC, END> piece;
    piece.load((const T *)g.weight, c, g.dim);
#pragma unroll
    for (int e = 0; e < VEC; ++e) w[e] = piece.get(e);
  }
}

// 1 / sqrt(mean + eps) of a row's squares, whose sum over the row `sum` forms of values times a factor (all lanes of a row take the same way).  Where the
// sum leaves fp32's range, of values times 2^-80 once more.  Where mean + eps is below 2^-100, so that squares below fp32's normal numbers (each off by up to
// 2^-126, were they left out) would be seen, of values times 2^100: they are at most 2^-50 sqrt(dim), and their squares 2^-98 at least.  1 / rms itself is above
// fp32's range below 2^-128: the row's values times `by` and the result `of_scaled` are in it, and rstd = by * of_scaled where that has a number.
struct RowScale {
  float by, of_scaled;  // h * rstd = (h * by) * of_scaled; by is 1 or 2^100
};
template <typename Sum>
__device__ __forceinline__ RowScale row_rstd(Sum sum, float inv_dim, float eps) {
  float sq = sum(1.0f);
  const float mean = __builtin_fmaf(sq, inv_dim, eps);
  if (mean < 0x1p-100f) {
    sq = sum(0x1p100f);
    return {0x1p100f, 1.0f / sqrtf(__builtin_fmaf(sq, inv_dim, eps * 0x1p100f * 0x1p100f))};
  }
  if (sq < INFINITY || sq != sq) return {1.0f, 1.0f / sqrtf(mean)};
  sq = sum(0x1p-80f);
  return {1.0f, 0x1p-80f / sqrtf(sq * inv_dim)};  // (eps is nothing beside it)
}

// x + residual, rounded once to T.
template <typename T, int N, RowEnd END>
__device__ __forceinline__ void add_rounded(RowPiece<T, N, END> &x, const RowPiece<T, N, END> &residual) {
  float h[N];
#pragma unroll
  for (int e = 0; e < N; ++e) h[e] = x.get(e) + residual.get(e);
  x.set(h);
}

// (No __restrict__: sum may be x or residual, y may be x.)
template <typename T, int LANES, int ITEMS, RowEnd END, bool E4M3>
__global__ __launch_bounds__(kRmsThreads<LANES>) void rms_kernel(RmsArgs g) {
  __shared__ float room[LANES > kWave ? LANES / kWave : 1];
  constexpr int VEC = 16 / (int)sizeof(T), kGroups = kRmsThreads<LANES> / LANES;
  typedef RowPiece<T, VEC, END> P;
  const uint32_t lane = threadIdx.x % LANES;
  float w[ITEMS][VEC];
#pragma unroll
  for (int it = 0; it < ITEMS; ++it) load_weights<T, VEC, END>(w[it], g, (it * LANES + lane) * VEC);
  const float inv_dim = 1.0f / (float)g.dim;
  for (uint64_t row = (uint64_t)blockIdx.x * kGroups + threadIdx.x / LANES; row < g.n; row += (uint64_t)gridDim.x * kGroups) {
    const T *x = (const T *)g.x + row * g.x_stride;
    P p[ITEMS];
#pragma unroll
    for (int it = 0; it < ITEMS; ++it) p[it].load(x, (it * LANES + lane) * VEC, g.dim);
    if (g.residual) {
      const T *residual = (const T *)g.residual + row * g.residual_stride;
      P r[ITEMS];
#pragma unroll
      for (int it = 0; it < ITEMS; ++it) r[it].load(residual, (it * LANES + lane) * VEC, g.dim);
#pragma unroll
      for (int it = 0; it < ITEMS; ++it) add_rounded(p[it], r[it]);
      if (g.sum) {
        T *sum = (T *)g.sum + row * g.sum_stride;
#pragma unroll
        for (int it = 0; it < ITEMS; ++it) p[it].store(sum, (it * LANES + lane) * VEC, g.dim);
      }
    }
    const RowScale scale_of = row_rstd(
        [&](float by) {
          float sq = 0.0f;
#pragma unroll
          for (int it = 0; it < ITEMS; ++it)
#pragma unroll
            for (int e = 0; e < VEC; ++e) sq = __builtin_fmaf(p[it].get(e) * by, p[it].get(e) * by, sq);
          return row_sum<LANES>(sq, room);
        },
        inv_dim, g.eps);
    const float rstd = scale_of.of_scaled;
    if (lane == 0 && g.rstd) g.rstd[row] = scale_of.by * rstd;
    if (scale_of.by != 1.0f) {  // (exact: tiny values, of types with fp32's range, or zeros)
#pragma unroll
      for (int it = 0; it < ITEMS; ++it) {
        float v[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) v[e] = p[it].get(e) * scale_of.by;
        p[it].set(v);
      }
    }
    if constexpr (!E4M3) {
      T *y = (T *)g.y + row * g.y_stride;
#pragma unroll
      for (int it = 0; it < ITEMS; ++it) {
        float v[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) v[e] = p[it].get(e) * rstd * w[it][e];
        P o;
        o.set(v);
        o.store(y, (it * LANES + lane) * VEC, g.dim);
      }
    } else {
      uint8_t *y = (uint8_t *)g.y + row * g.y_stride;
      float *scales = g.scales + row * g.scale_stride;
      float v[ITEMS][VEC], most[ITEMS], whole = 0.0f;
#pragma unroll
      for (int it = 0; it < ITEMS; ++it) {
        most[it] = 0.0f;
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          v[it][e] = p[it].get(e) * rstd * w[it][e];
          most[it] = fmaxf(most[it], fabsf(v[it][e]));
        }
        whole = fmaxf(whole, most[it]);
      }
      if (g.group == 0) whole = row_max<LANES>(whole, room);
#pragma unroll
      for (int it = 0; it < ITEMS; ++it) {
        const uint32_t c = (it * LANES + lane) * VEC;
        const float scale = fmaxf(g.group ? lanes_max(most[it], g.group / VEC) : whole, kSmallestMax) / kE4m3Max;
        if (g.group ? c < g.dim && c % g.group == 0 : c == 0) scales[g.group ? c / g.group : 0] = scale;
        store_codes(v[it], scale, y, c, g.dim);
      }
    }
  }
}

// Rows longer than a workgroup's registers: passes over the row (all but the first find it in the L2), kept sums included: each lane
// reads again what it wrote itself.
template <typename T, bool E4M3>
__global__ __launch_bounds__(1024) void rms_long_kernel(RmsArgs g) {
  __shared__ float room[1024 / kWave];
  constexpr int VEC = 16 / (int)sizeof(T);
  typedef RowPiece<T, VEC> P;
  const float inv_dim = 1.0f / (float)g.dim;
  const uint32_t pieces = (g.dim + VEC - 1) / VEC, rounds = (pieces + 1023) / 1024;
  for (uint64_t row = blockIdx.x; row < g.n; row += gridDim.x) {
    const T *x = (const T *)g.x + row * g.x_stride, *residual = g.residual ? (const T *)g.residual + row * g.residual_stride : nullptr;
    T *sum = g.sum ? (T *)g.sum + row * g.sum_stride : nullptr;
    // h, from the rows as they came (KEPT: from the sums that are kept, which may have taken their place)
    const auto piece = [&](uint32_t c, bool kept) {
      P p;
      if (kept && sum) {
        p.load(sum, c, g.dim);
        return p;
      }
      p.load(x, c, g.dim);
      if (residual) {
        P r;
        r.load(residual, c, g.dim);
        add_rounded(p, r);
        if (sum) p.store(sum, c, g.dim);
      }
      return p;
    };
    const RowScale scale_of = row_rstd(
        [&](float by) {
          float sq = 0.0f;
          for (uint32_t c = threadIdx.x * VEC; c < g.dim; c += 1024 * VEC) {
            const P p = piece(c, by != 1.0f);
#pragma unroll
            for (int e = 0; e < VEC; ++e) sq = __builtin_fmaf(p.get(e) * by, p.get(e) * by, sq);
          }
          return row_sum<1024>(sq, room);
        },
        inv_dim, g.eps);
    if (threadIdx.x == 0 && g.rstd) g.rstd[row] = scale_of.by * scale_of.of_scaled;
    const auto value = [&](const P &p, uint32_t c, int e) {
      return p.get(e) * scale_of.by * scale_of.of_scaled * (g.weight && c + e < g.dim ? load_param<T>(g.weight, g.weight_f32, c + e) : 1.0f);
    };
    if constexpr (!E4M3) {
      T *y = (T *)g.y + row * g.y_stride;
      for (uint32_t c = threadIdx.x * VEC; c < g.dim; c += 1024 * VEC) {
        P p = piece(c, true);
        float v[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) v[e] = value(p, c, e);
        p.set(v);
        p.store(y, c, g.dim);
      }
    } else {
      uint8_t *y = (uint8_t *)g.y + row * g.y_stride;
      float *scales = g.scales + row * g.scale_stride, whole = 0.0f;
      if (g.group == 0) {
        for (uint32_t c = threadIdx.x * VEC; c < g.dim; c += 1024 * VEC) {
          const P p = piece(c, true);
#pragma unroll
          for (int e = 0; e < VEC; ++e) whole = fmaxf(whole, fabsf(value(p, c, e)));
        }
        whole = row_max<1024>(whole, room);
      }
      for (uint32_t round = 0; round < rounds; ++round) {  // (all lanes take part in a group's maximum)
        const uint32_t c = (round * 1024 + threadIdx.x) * VEC;
        const bool in = c < g.dim;
        float v[VEC], most = 0.0f;
        P p;
        if (in) p = piece(c, true);
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          v[e] = in ? value(p, c, e) : 0.0f;
          most = fmaxf(most, fabsf(v[e]));
        }
        const float scale = fmaxf(g.group ? lanes_max(most, g.group / VEC) : whole, kSmallestMax) / kE4m3Max;
        if (in && (g.group ? c % g.group == 0 : c == 0)) scales[g.group ? c / g.group : 0] = scale;
        if (in) store_codes(v, scale, y, c, g.dim);
      }
    }
  }
}

// PARAMS: the gradient of w is wanted.  (dx may be dy or dsum.)
template <typename T, int LANES, int ITEMS, RowEnd END, bool PARAMS>
__global__ __launch_bounds__(kRmsThreads<LANES>) void rms_grad_kernel(RmsArgs g) {
  __shared__ float room[LANES > kWave ? LANES / kWave : 1];
  constexpr int VEC = 16 / (int)sizeof(T), kGroups = kRmsThreads<LANES> / LANES;
  typedef RowPiece<T, VEC, END> P;
  const uint32_t lane = threadIdx.x % LANES;
  float w[ITEMS][VEC], dw[ITEMS][VEC];
#pragma unroll
  for (int it = 0; it < ITEMS; ++it) {
    load_weights<T, VEC, END>(w[it], g, (it * LANES + lane) * VEC);
#pragma unroll
    for (int e = 0; e < VEC; ++e) dw[it][e] = 0.0f;
  }
  const float inv_dim = 1.0f / (float)g.dim;
  for (uint64_t row = (uint64_t)blockIdx.x * kGroups + threadIdx.x / LANES; row < g.n; row += (uint64_t)gridDim.x * kGroups) {
    const T *h = (const T *)g.x + row * g.x_stride, *dy = (const T *)g.dy + row * g.dy_stride;
    const float rstd = g.rstd[row];
    P ph[ITEMS], pd[ITEMS], ps[ITEMS];
#pragma unroll
    for (int it = 0; it < ITEMS; ++it) ph[it].load(h, (it * LANES + lane) * VEC, g.dim), pd[it].load(dy, (it * LANES + lane) * VEC, g.dim);
    if (g.residual) {
      const T *dsum = (const T *)g.residual + row * g.residual_stride;
#pragma unroll
      for (int it = 0; it < ITEMS; ++it) ps[it].load(dsum, (it * LANES + lane) * VEC, g.dim);
    }
    float along = 0.0f;
#pragma unroll
    for (int it = 0; it < ITEMS; ++it)
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const float xh = ph[it].get(e) * rstd, d = pd[it].get(e);
        along = __builtin_fmaf(d * w[it][e], xh, along);
        if constexpr (PARAMS) dw[it][e] = __builtin_fmaf(d, xh, dw[it][e]);
      }
    const float mean = row_sum<LANES>(along, room) * inv_dim;
    T *dx = (T *)g.y + row * g.y_stride;
#pragma unroll
    for (int it = 0; it < ITEMS; ++it) {
      float v[VEC];
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const float xh = ph[it].get(e) * rstd, a = pd[it].get(e) * w[it][e], d = __builtin_fmaf(-xh, mean, a);
        v[e] = g.residual ? __builtin_fmaf(rstd, d, ps[it].get(e)) : rstd * d;
      }
      P o;
      o.set(v);
      o.store(dx, (it * LANES + lane) * VEC, g.dim);
    }
  }
  if constexpr (PARAMS) {
    // the groups' sums one after the other: those of a wavefront by lane exchanges, the wavefronts' in LDS
    constexpr int kWaves = kRmsThreads<LANES> / kWave;
    __shared__ float acc[LANES <= kWave ? ITEMS * VEC * LANES : 1];
    float *out = g.partial + (uint64_t)blockIdx.x * g.dim;
    if constexpr (LANES <= kWave) {
      for (int wave = 0; wave < kWaves; ++wave) {
        if ((int)threadIdx.x / kWave == wave) {
#pragma unroll
          for (int it = 0; it < ITEMS; ++it)
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
              float v = dw[it][e];
              if constexpr (LANES == 16) {
                const LanePair p = lane_pair<true>(__float_as_uint(v));
                v = __uint_as_float(p.low) + __uint_as_float(p.high);
              }
              if constexpr (LANES <= 32) {
                const LanePair p = lane_pair<false>(__float_as_uint(v));
                v = __uint_as_float(p.low) + __uint_as_float(p.high);
              }
              const int at = (it * LANES + (int)lane) * VEC + e;
              if (threadIdx.x % kWave < LANES) acc[at] = wave == 0 ? v : acc[at] + v;
            }
        }
        __syncthreads();
      }
      for (uint32_t c = threadIdx.x; c < g.dim; c += kRmsThreads<LANES>) out[c] = acc[c];
    } else {
#pragma unroll
      for (int it = 0; it < ITEMS; ++it)
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          const uint32_t c = (it * LANES + lane) * VEC + e;
          if (c < g.dim) out[c] = dw[it][e];
        }
    }
  }
}

template <typename T>
__global__ __launch_bounds__(1024) void rms_grad_long_kernel(RmsArgs g) {
  __shared__ float room[1024 / kWave];
  constexpr int VEC = 16 / (int)sizeof(T);
  typedef RowPiece<T, VEC> P;
  const float inv_dim = 1.0f / (float)g.dim;
  float *out = g.partial ? g.partial + (uint64_t)blockIdx.x * g.dim : nullptr;
  for (uint64_t row = blockIdx.x; row < g.n; row += gridDim.x) {
    const T *h = (const T *)g.x + row * g.x_stride, *dy = (const T *)g.dy + row * g.dy_stride;
    const T *dsum = g.residual ? (const T *)g.residual + row * g.residual_stride : nullptr;
    T *dx = (T *)g.y + row * g.y_stride;
    const float rstd = g.rstd[row];
    const auto weight = [&](uint32_t c) { return g.weight && c < g.dim ? load_param<T>(g.weight, g.weight_f32, c) : 1.0f; };
    float along = 0.0f;
    for (uint32_t c = threadIdx.x * VEC; c < g.dim; c += 1024 * VEC) {
      P ph, pd;
      ph.load(h, c, g.dim), pd.load(dy, c, g.dim);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const float xh = ph.get(e) * rstd, d = pd.get(e);
        along = __builtin_fmaf(d * weight(c + e), xh, along);
        // the lane's own columns of the workgroup's own partial sums
        if (out && c + e < g.dim) out[c + e] = row == blockIdx.x ? d * xh : __builtin_fmaf(d, xh, out[c + e]);
      }
    }
    const float mean = row_sum<1024>(along, room) * inv_dim;
    for (uint32_t c = threadIdx.x * VEC; c < g.dim; c += 1024 * VEC) {
      P ph, pd, ps;
      ph.load(h, c, g.dim), pd.load(dy, c, g.dim);
      if (dsum) ps.load(dsum, c, g.dim);
      float v[VEC];
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const float xh = ph.get(e) * rstd, a = pd.get(e) * weight(c + e), d = __builtin_fmaf(-xh, mean, a);
        v[e] = dsum ? __builtin_fmaf(rstd, d, ps.get(e)) : rstd * d;
      }
      pd.set(v);
      pd.store(dx, c, g.dim);
    }
  }
}

// The partial sums of 64 columns in the order of the workgroups: 16 runs of them, 16 parts of a run on their way at a time, then the runs.
template <typename T>
__global__ __launch_bounds__(1024) void rms_grad_sum_kernel(const float *__restrict__ partial, uint32_t parts, uint32_t dim, void *dweight, bool f32) {
  __shared__ float runs[16][64];
  const uint32_t lane = threadIdx.x % 64, run = threadIdx.x / 64, c = blockIdx.x * 64 + lane;
  float sum = 0.0f;
  if (c < dim) {
    const uint32_t end = (run + 1) * parts / 16;
    for (uint32_t p = run * parts / 16; p < end; p += 16) {
      float v[16];
#pragma unroll
      for (uint32_t u = 0; u < 16; ++u) v[u] = p + u < end ? partial[(uint64_t)(p + u) * dim + c] : 0.0f;
#pragma unroll
      for (uint32_t u = 0; u < 16; ++u) sum += v[u];
    }
  }
  runs[run][lane] = sum;
  __syncthreads();
  if (run != 0 || c >= dim) return;
  sum = 0.0f;
#pragma unroll
  for (int r = 0; r < 16; ++r) sum += runs[r][lane];
  store_param<T>(dweight, f32, c, sum);
}

static uint32_t rms_parts(uint64_t n) { return (uint32_t)(n / 4 < 1 ? 1 : n / 4 < kRmsParts ? n / 4 : kRmsParts); }

// Launches one of the kernels above: lanes and pieces to a lane that leave few of them without work, and that hold a group that shares a
// scale side by side.
enum RmsKind { kNorm, kNormE4m3, kGrad };

template <typename T, RmsKind KIND>
static void launch_rms(const RmsArgs &g, hipStream_t st) {
  constexpr uint32_t VEC = 16 / sizeof(T);
  const auto run_as = [&](auto lanes, auto items, auto whole) {
    constexpr int L = decltype(lanes)::value, ITEMS = decltype(items)::value;
    constexpr RowEnd END = decltype(whole)::value ? kWholePieces : L <= kWave ? kShifted : kByElement;
    constexpr int kGroups = kRmsThreads<L> / L;
    const uint64_t want = (g.n + kGroups - 1) / kGroups;
    const uint32_t blocks = (uint32_t)(want < kRmsBlocks ? want : kRmsBlocks);
    if constexpr (KIND == kGrad) {
      if (g.partial)
        rms_grad_kernel<T, L, ITEMS, END, true><<<rms_parts(g.n), kRmsThreads<L>, 0, st>>>(g);
      else
        rms_grad_kernel<T, L, ITEMS, END, false><<<blocks, kRmsThreads<L>, 0, st>>>(g);
    } else {
      rms_kernel<T, L, ITEMS, END, KIND == kNormE4m3><<<blocks, kRmsThreads<L>, 0, st>>>(g);
    }
  };
  const auto run = [&](auto lanes, auto items) {
    if (g.dim % VEC == 0)
      run_as(lanes, items, std::true_type());
    else
      run_as(lanes, items, std::false_type());
  };
  const std::integral_constant<int, 1> i1;
  const std::integral_constant<int, 2> i2;
  const std::integral_constant<int, 3> i3;
  const std::integral_constant<int, 4> i4;
  const std::integral_constant<int, 16> l16;
  const std::integral_constant<int, 32> l32;
  const std::integral_constant<int, 64> l64;
  const std::integral_constant<int, 256> l256;
  const std::integral_constant<int, 512> l512;
  const uint32_t pieces = (g.dim + VEC - 1) / VEC;
  const bool side_by_side = KIND != kNormE4m3 || g.group <= 16 * VEC;  // within 16 lanes
  if (pieces <= 16 && side_by_side)
    run(l16, i1);
  else if (pieces <= 32 && side_by_side)
    run(l16, i2);
  else if (pieces <= 64)
    run(l32, i2);
  else if (pieces <= 96)
    run(l32, i3);
  else if (pieces <= 128)
    run(l32, i4);
  else if (pieces <= 192)
    run(l64, i3);
  else if (pieces <= 256)
    run(l64, i4);
  else if (pieces <= 512)
    run(l256, i2);
  else if (pieces <= 768)
    run(l256, i3);
  else if (pieces <= 1024)
    run(l256, i4);
  else if (pieces <= 1536)
    run(l512, i3);
  else if (pieces <= 2048)
    run(l512, i4);
  else {
    const uint32_t rows = (uint32_t)(g.n < kRmsBlocks ? g.n : kRmsBlocks);
    if constexpr (KIND == kGrad)
      rms_grad_long_kernel<T><<<g.partial ? rms_parts(g.n) : rows, 1024, 0, st>>>(g);
    else
      rms_long_kernel<T, KIND == kNormE4m3><<<rows, 1024, 0, st>>>(g);
  }
}

template <RmsKind KIND>
static ann_status launch_rms_typed(uint32_t type, const RmsArgs &g, hipStream_t st) {
  if (type == ANN_F32)
    launch_rms<float, KIND>(g, st);
  else if (type == ANN_F16)
    launch_rms<f16_t, KIND>(g, st);
  else
    launch_rms<bf16_t, KIND>(g, st);
  ANN_HIP(hipGetLastError());
  return ANN_OK;
}

static ann_status check_rms(const char *what, uint64_t n, uint32_t dim, uint32_t type, uint32_t weight_type, bool weight) {
  if (type > ANN_BF16) return fail(ANN_EINVAL, "%s: unknown type %u", what, type);
  if (weight && weight_type != type && weight_type != ANN_F32)
    return fail(ANN_EINVAL, "%s: weights are of the rows' type or ANN_F32, not %u", what, weight_type);
  if (dim == 0) return fail(ANN_EINVAL, "%s: dim == 0", what);
  if (dim > ANN_MAX_NORM_DIM) return fail(ANN_ECAPACITY, "%s: dim = %u exceeds ANN_MAX_NORM_DIM = %u", what, dim, ANN_MAX_NORM_DIM);
  if (n >= (1ull << 40)) return fail(ANN_ECAPACITY, "%s: n = %llu", what, (unsigned long long)n);
  return ANN_OK;
}

static ann_status check_rms_rows(const char *what, const RmsArgs &g) {
  if (!g.x || !g.y) return fail(ANN_EINVAL, "%s: NULL argument", what);
  if (g.sum && !g.residual) return fail(ANN_EINVAL, "%s: sum without residual", what);
  if (g.sum && g.sum == g.y) return fail(ANN_EINVAL, "%s: sum and y are the same rows", what);
  if (g.x_stride < g.dim || g.y_stride < g.dim || (g.residual && g.residual_stride < g.dim) || (g.sum && g.sum_stride < g.dim))
    return fail(ANN_EINVAL, "%s: a row stride is shorter than a row", what);
  if (!(g.eps >= 0.0f)) return fail(ANN_EINVAL, "%s: eps must not be negative", what);
  return ANN_OK;
}

}  // namespace ann

using namespace ann;

extern "C" ann_status ann_rms_norm(const void *x, uint64_t n, uint32_t dim, uint64_t x_stride, uint32_t type, const void *residual,
                                   uint64_t residual_stride, const void *weight, uint32_t weight_type, float eps, void *sum, uint64_t sum_stride,
                                   void *y, uint64_t y_stride, float *rstd, void *stream) {
  if (ann_status s = check_rms("ann_rms_norm", n, dim, type, weight_type, weight)) return s;
  if (n == 0) return ANN_OK;
  RmsArgs g = {};
  g.x = x, g.residual = residual, g.weight = weight, g.sum = sum, g.y = y, g.rstd = rstd, g.n = n, g.dim = dim, g.eps = eps;
  g.x_stride = x_stride, g.residual_stride = residual_stride, g.sum_stride = sum_stride, g.y_stride = y_stride, g.weight_f32 = weight_type == ANN_F32;
  if (ann_status s = check_rms_rows("ann_rms_norm", g)) return s;
  return launch_rms_typed<kNorm>(type, g, (hipStream_t)stream);
}

extern "C" ann_status ann_rms_norm_e4m3(const void *x, uint64_t n, uint32_t dim, uint64_t x_stride, uint32_t type, const void *residual,
                                        uint64_t residual_stride, const void *weight, uint32_t weight_type, float eps, void *sum,
                                        uint64_t sum_stride, uint8_t *y, uint64_t y_stride, uint32_t group, float *scales, uint64_t scale_stride,
                                        float *rstd, void *stream) {
  if (ann_status s = check_rms("ann_rms_norm_e4m3", n, dim, type, weight_type, weight)) return s;
  if (group != 0 && group != 32 && group != 64 && group != 128) return fail(ANN_EINVAL, "ann_rms_norm_e4m3: group = %u", group);
  if (n == 0) return ANN_OK;
  RmsArgs g = {};
  g.x = x, g.residual = residual, g.weight = weight, g.sum = sum, g.y = y, g.rstd = rstd, g.n = n, g.dim = dim, g.eps = eps;
  g.x_stride = x_stride, g.residual_stride = residual_stride, g.sum_stride = sum_stride, g.y_stride = y_stride, g.weight_f32 = weight_type == ANN_F32;
  g.group = group, g.scales = scales, g.scale_stride = scale_stride;
  if (ann_status s = check_rms_rows("ann_rms_norm_e4m3", g)) return s;
  if (!scales) return fail(ANN_EINVAL, "ann_rms_norm_e4m3: scales is NULL");
  if (y == x || y == residual) return fail(ANN_EINVAL, "ann_rms_norm_e4m3: y cannot take the place of its input");
  if (scale_stride < (group ? (dim + group - 1) / group : 1)) return fail(ANN_EINVAL, "ann_rms_norm_e4m3: scale_stride is shorter than a row's scales");
  return launch_rms_typed<kNormE4m3>(type, g, (hipStream_t)stream);
}

extern "C" uint64_t ann_rms_norm_backward_workspace(uint64_t n, uint32_t dim) { return n == 0 ? 0 : (uint64_t)rms_parts(n) * dim * sizeof(float); }

extern "C" ann_status ann_rms_norm_backward(const void *dy, uint64_t dy_stride, const void *h, uint64_t h_stride, uint64_t n, uint32_t dim,
                                            uint32_t type, const void *dsum, uint64_t dsum_stride, const void *weight, uint32_t weight_type,
                                            const float *rstd, void *dx, uint64_t dx_stride, void *dweight, void *workspace,
                                            uint64_t workspace_bytes, void *stream) {
  if (ann_status s = check_rms("ann_rms_norm_backward", n, dim, type, weight_type, weight || dweight)) return s;
  if (n && (!dy || !h || !rstd || !dx)) return fail(ANN_EINVAL, "ann_rms_norm_backward: NULL argument");
  if (n && (h_stride < dim || dy_stride < dim || dx_stride < dim || (dsum && dsum_stride < dim)))
    return fail(ANN_EINVAL, "ann_rms_norm_backward: a row stride is shorter than a row");
  const uint64_t need = dweight ? ann_rms_norm_backward_workspace(n, dim) : 0;
  if (need && !workspace) return fail(ANN_EINVAL, "ann_rms_norm_backward: workspace is NULL");
  if (workspace_bytes < need)
    return fail(ANN_EINVAL, "ann_rms_norm_backward: workspace of %llu bytes, %llu are needed", (unsigned long long)workspace_bytes,
                (unsigned long long)need);
  if (need && (uintptr_t)workspace % 16) return fail(ANN_EINVAL, "ann_rms_norm_backward: workspace is not aligned to 16 bytes");
  const hipStream_t st = (hipStream_t)stream;
  RmsArgs g = {};
  g.x = h, g.dy = dy, g.residual = dsum, g.weight = weight, g.y = dx, g.rstd = (float *)rstd, g.partial = dweight ? (float *)workspace : nullptr;
  g.n = n, g.x_stride = h_stride, g.dy_stride = dy_stride, g.residual_stride = dsum_stride, g.y_stride = dx_stride, g.dim = dim;
  g.weight_f32 = weight_type == ANN_F32;
  if (n)
    if (ann_status s = launch_rms_typed<kGrad>(type, g, st)) return s;
  if (!dweight) return ANN_OK;
  const uint32_t parts = n ? rms_parts(n) : 0, grid = (dim + 63) / 64;
  if (type == ANN_F16)
    rms_grad_sum_kernel<f16_t><<<grid, 1024, 0, st>>>(g.partial, parts, dim, dweight, g.weight_f32);
  else if (type == ANN_BF16)
    rms_grad_sum_kernel<bf16_t><<<grid, 1024, 0, st>>>(g.partial, parts, dim, dweight, g.weight_f32);
  else
    rms_grad_sum_kernel<float><<<grid, 1024, 0, st>>>(g.partial, parts, dim, dweight, true);
  ANN_HIP(hipGetLastError());
  return ANN_OK;
}
