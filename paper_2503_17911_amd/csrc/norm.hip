// Layer norm of the rows of a matrix and its gradients.
//
//   y = (x - mean) * rstd * w + b,  rstd = 1 / sqrt(mean((x - mean)^2) + eps)
//   dx = rstd * (a - mean(a) - xh * mean(a * xh)),  a = dy * w,  xh = (x - mean) * rstd
//   dw = sum over rows of dy * xh,  db = sum over rows of dy
//
// Bound by memory: x (and dy) are read once and stay in registers, as the pieces
// that were loaded, while the row's sums are formed; every sum is fp32.  The
// variance is that of the centred values in registers, not a difference of two
// large sums.  A row belongs to LANES lanes of a wavefront, or to a workgroup of
// 256 or 512 lanes (1,024 lanes have 128 registers each, too few for the pieces and both gradients); each lane holds up to
// kItems pieces.  Groups walk over rows, so that weights are read once per group, and, in the backward pass, the
// gradients of w and b collect in registers: one partial sum per workgroup goes
// to the workspace, a second kernel adds them in a fixed order (no atomics: the
// result does not depend on timing).  Measured: 200,000 x 960 fp32 forward 292 us
// (5.3 TB/s; a large copy reaches 5.1), 80,000 x 768 bf16 backward 76 us (4.9 TB/s), of
// which 4.6 are the second kernel; 5,003 x 100 fp16 backward 15 us, all of it
// latency: loads, sums, two launches.
#include <type_traits>

#include "ann_internal.hpp"
#include "device_utils.hpp"
#include "scalar_types.hpp"

namespace ann {

constexpr int kItems = 4;              // pieces of a row to a lane
constexpr uint32_t kNormBlocks = 2048; // workgroups of the forward pass at most: 8 of 256 lanes per compute unit
constexpr uint32_t kNormParts = 512;   // partial sums of the weights' gradient at most: two workgroups per compute unit

__device__ __forceinline__ float wave_sum(float v, int lanes) {
  if (lanes >= 2) v += __int_as_float(dpp_i32<kDppQuadXor1>(__float_as_int(v)));
  if (lanes >= 4) v += __int_as_float(dpp_i32<kDppQuadXor2>(__float_as_int(v)));
  if (lanes >= 8) v += __int_as_float(dpp_i32<kDppRowHalfMirror>(__float_as_int(v)));
  if (lanes >= 16) v += __int_as_float(dpp_i32<kDppRowMirror>(__float_as_int(v)));
  if (lanes >= 32) {
    const LanePair p = lane_pair<true>(__float_as_uint(v));
    v = __uint_as_float(p.low) + __uint_as_float(p.high);
  }
  if (lanes >= 64) {
    const LanePair p = lane_pair<false>(__float_as_uint(v));
    v = __uint_as_float(p.low) + __uint_as_float(p.high);
  }
  return v;
}

// Sums of a and b over the LANES lanes that share a row; every one of them gets both.
template <int LANES>
__device__ __forceinline__ void row_sums(float &a, float &b, float2 *room) {
  a = wave_sum(a, LANES < kWave ? LANES : kWave);
  b = wave_sum(b, LANES < kWave ? LANES : kWave);
  if constexpr (LANES > kWave) {
    __syncthreads();  // the last row's sums have been read
    if (threadIdx.x % kWave == 0) room[threadIdx.x / kWave] = make_float2(a, b);
    __syncthreads();
    a = 0.0f, b = 0.0f;
#pragma unroll
    for (int w = 0; w < LANES / kWave; ++w) a += room[w].x, b += room[w].y;
  }
}

struct NormArgs {
  const void *x, *dy, *weight, *bias;
  void *y;                       // forward: y; backward: dx
  float *mean, *rstd, *partial;  // partial: [workgroups][2][dim]
  uint64_t n, x_stride, dy_stride, y_stride;
  uint32_t dim;
  float eps;
  bool weight_f32;
};

template <int LANES>
constexpr int kNormThreads = LANES > 256 ? LANES : 256;

// VEC elements to a piece.  (x and y may be the same rows: no __restrict__.)
template <typename T, int VEC, int LANES>
__global__ __launch_bounds__(kNormThreads<LANES>) void norm_kernel(NormArgs g) {
  __shared__ float2 room[LANES > kWave ? LANES / kWave : 1];
  typedef Piece<T, VEC> P;
  constexpr int kGroups = kNormThreads<LANES> / LANES;
  const uint32_t lane = threadIdx.x % LANES;
  float w[kItems][VEC], b[kItems][VEC];
#pragma unroll
  for (int it = 0; it < kItems; ++it)
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      const uint32_t c = (it * LANES + lane) * VEC + e;
      w[it][e] = g.weight && c < g.dim ? load_param<T>(g.weight, g.weight_f32, c) : 1.0f;
      b[it][e] = g.bias && c < g.dim ? load_param<T>(g.bias, g.weight_f32, c) : 0.0f;
    }
  const float inv = 1.0f / (float)g.dim;
  for (uint64_t row = (uint64_t)blockIdx.x * kGroups + threadIdx.x / LANES; row < g.n; row += (uint64_t)gridDim.x * kGroups) {
    const T *x = (const T *)g.x + row * g.x_stride;
    P p[kItems];
    float sum = 0.0f, none = 0.0f;
#pragma unroll
    for (int it = 0; it < kItems; ++it) {
      const uint32_t c = (it * LANES + lane) * VEC;
      if (c < g.dim) {
        p[it] = *(const P *)(x + c);
      } else {
#pragma unroll
        for (int e = 0; e < VEC; ++e) p[it].v[e] = (T)0.0f;
      }
    }
#pragma unroll
    for (int it = 0; it < kItems; ++it)
#pragma unroll
      for (int e = 0; e < VEC; ++e) sum += to_f32(p[it].v[e]);
    row_sums<LANES>(sum, none, room);
    const float mean = sum * inv;
    float sq = 0.0f;
#pragma unroll
    for (int it = 0; it < kItems; ++it) {
      const bool in = (it * LANES + lane) * VEC < g.dim;
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const float v = in ? to_f32(p[it].v[e]) - mean : 0.0f;
        sq = __builtin_fmaf(v, v, sq);
      }
    }
    row_sums<LANES>(sq, none, room);
    const float rstd = 1.0f / sqrtf(__builtin_fmaf(sq, inv, g.eps));
    if (lane == 0) {
      if (g.mean) g.mean[row] = mean;
      if (g.rstd) g.rstd[row] = rstd;
    }
    T *y = (T *)g.y + row * g.y_stride;
#pragma unroll
    for (int it = 0; it < kItems; ++it) {
      const uint32_t c = (it * LANES + lane) * VEC;
      if (c < g.dim) {
        P o;
#pragma unroll
        for (int e = 0; e < VEC; ++e) o.v[e] = from_f32<T>(__builtin_fmaf((to_f32(p[it].v[e]) - mean) * rstd, w[it][e], b[it][e]));
        *(P *)(y + c) = o;
      }
    }
  }
}

// Rows longer than a workgroup's registers: three passes over the row (the second and third find it in the L2).
template <typename T>
__global__ __launch_bounds__(1024) void norm_long_kernel(NormArgs g) {
  __shared__ float2 room[1024 / kWave];
  const float inv = 1.0f / (float)g.dim;
  for (uint64_t row = blockIdx.x; row < g.n; row += gridDim.x) {
    const T *x = (const T *)g.x + row * g.x_stride;
    T *y = (T *)g.y + row * g.y_stride;
    float sum = 0.0f, sq = 0.0f, none = 0.0f;
    for (uint32_t c = threadIdx.x; c < g.dim; c += 1024) sum += to_f32(x[c]);
    row_sums<1024>(sum, none, room);
    const float mean = sum * inv;
    for (uint32_t c = threadIdx.x; c < g.dim; c += 1024) {
      const float v = to_f32(x[c]) - mean;
      sq = __builtin_fmaf(v, v, sq);
    }
    row_sums<1024>(sq, none, room);
    const float rstd = 1.0f / sqrtf(__builtin_fmaf(sq, inv, g.eps));
    if (threadIdx.x == 0) {
      if (g.mean) g.mean[row] = mean;
      if (g.rstd) g.rstd[row] = rstd;
    }
    for (uint32_t c = threadIdx.x; c < g.dim; c += 1024) {
      const float w = g.weight ? load_param<T>(g.weight, g.weight_f32, c) : 1.0f;
      const float b = g.bias ? load_param<T>(g.bias, g.weight_f32, c) : 0.0f;
      y[c] = from_f32<T>(__builtin_fmaf((to_f32(x[c]) - mean) * rstd, w, b));
    }
  }
}

// PARAMS: the gradients of w and b are wanted.
template <typename T, int VEC, int LANES, bool PARAMS>
__global__ __launch_bounds__(kNormThreads<LANES>) void norm_grad_kernel(NormArgs g) {
  __shared__ float2 room[LANES > kWave ? LANES / kWave : 1];
  typedef Piece<T, VEC> P;
  constexpr int kGroups = kNormThreads<LANES> / LANES;
  const uint32_t lane = threadIdx.x % LANES;
  float w[kItems][VEC], dw[kItems][VEC], db[kItems][VEC];
#pragma unroll
  for (int it = 0; it < kItems; ++it)
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      const uint32_t c = (it * LANES + lane) * VEC + e;
      w[it][e] = g.weight && c < g.dim ? load_param<T>(g.weight, g.weight_f32, c) : 1.0f;
      dw[it][e] = 0.0f, db[it][e] = 0.0f;
    }
  const float inv = 1.0f / (float)g.dim;
  for (uint64_t row = (uint64_t)blockIdx.x * kGroups + threadIdx.x / LANES; row < g.n; row += (uint64_t)gridDim.x * kGroups) {
    const T *x = (const T *)g.x + row * g.x_stride, *dy = (const T *)g.dy + row * g.dy_stride;
    const float mean = g.mean[row], rstd = g.rstd[row];
    P px[kItems], pd[kItems];
#pragma unroll
    for (int it = 0; it < kItems; ++it) {
      const uint32_t c = (it * LANES + lane) * VEC;
      if (c < g.dim) px[it] = *(const P *)(x + c), pd[it] = *(const P *)(dy + c);
    }
    float sa = 0.0f, sax = 0.0f;
#pragma unroll
    for (int it = 0; it < kItems; ++it)
      if ((it * LANES + lane) * VEC < g.dim) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          const float xh = (to_f32(px[it].v[e]) - mean) * rstd, d = to_f32(pd[it].v[e]), a = d * w[it][e];
          sa += a;
          sax = __builtin_fmaf(a, xh, sax);
          if constexpr (PARAMS) {
            dw[it][e] = __builtin_fmaf(d, xh, dw[it][e]);
            db[it][e] += d;
          }
        }
      }
    row_sums<LANES>(sa, sax, room);
    const float ma = sa * inv, max_ = sax * inv;
    T *dx = (T *)g.y + row * g.y_stride;
#pragma unroll
    for (int it = 0; it < kItems; ++it) {
      const uint32_t c = (it * LANES + lane) * VEC;
      if (c < g.dim) {
        P o;
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          const float xh = (to_f32(px[it].v[e]) - mean) * rstd, a = to_f32(pd[it].v[e]) * w[it][e];
          o.v[e] = from_f32<T>(rstd * (a - __builtin_fmaf(xh, max_, ma)));
        }
        *(P *)(dx + c) = o;
      }
    }
  }
  if constexpr (PARAMS) {
    // the groups' sums one after the other: those of a wavefront by lane exchanges, the wavefronts' in LDS
    constexpr int kWaves = kNormThreads<LANES> / kWave;
    __shared__ float acc[LANES <= kWave ? kItems * VEC * LANES : 1];
    float *out = g.partial + (uint64_t)blockIdx.x * 2 * g.dim;
    for (int which = 0; which < 2; ++which) {
      if constexpr (LANES <= kWave) {
        for (int wave = 0; wave < kWaves; ++wave) {
          if ((int)threadIdx.x / kWave == wave) {
#pragma unroll
            for (int it = 0; it < kItems; ++it)
#pragma unroll
              for (int e = 0; e < VEC; ++e) {
                float v = which ? db[it][e] : dw[it][e];
                if constexpr (LANES == 16) {
                  LanePair p = lane_pair<true>(__float_as_uint(v));
                  v = __uint_as_float(p.low) + __uint_as_float(p.high);
                  p = lane_pair<false>(__float_as_uint(v));
                  v = __uint_as_float(p.low) + __uint_as_float(p.high);
                }
                const int at = (it * LANES + (int)lane) * VEC + e;
                if (threadIdx.x % kWave < LANES) acc[at] = wave == 0 ? v : acc[at] + v;
              }
          }
          __syncthreads();
        }
        for (uint32_t c = threadIdx.x; c < g.dim; c += kNormThreads<LANES>) out[which * g.dim + c] = acc[c];
        __syncthreads();
      } else {
#pragma unroll
        for (int it = 0; it < kItems; ++it)
#pragma unroll
          for (int e = 0; e < VEC; ++e) {
            const uint32_t c = (it * LANES + lane) * VEC + e;
            if (c < g.dim) out[which * g.dim + c] = which ? db[it][e] : dw[it][e];
          }
      }
    }
  }
}

template <typename T>
__global__ __launch_bounds__(1024) void norm_grad_long_kernel(NormArgs g) {
  __shared__ float2 room[1024 / kWave];
  const float inv = 1.0f / (float)g.dim;
  float *out = g.partial ? g.partial + (uint64_t)blockIdx.x * 2 * g.dim : nullptr;
  for (uint64_t row = blockIdx.x; row < g.n; row += gridDim.x) {
    const T *x = (const T *)g.x + row * g.x_stride, *dy = (const T *)g.dy + row * g.dy_stride;
    T *dx = (T *)g.y + row * g.y_stride;
    const float mean = g.mean[row], rstd = g.rstd[row];
    float sa = 0.0f, sax = 0.0f;
    for (uint32_t c = threadIdx.x; c < g.dim; c += 1024) {
      const float xh = (to_f32(x[c]) - mean) * rstd, d = to_f32(dy[c]);
      const float a = g.weight ? d * load_param<T>(g.weight, g.weight_f32, c) : d;
      sa += a;
      sax = __builtin_fmaf(a, xh, sax);
      if (out) {  // the lane's own columns of the workgroup's own partial sums
        const bool first = row == blockIdx.x;
        out[c] = first ? d * xh : __builtin_fmaf(d, xh, out[c]);
        out[g.dim + c] = first ? d : out[g.dim + c] + d;
      }
    }
    row_sums<1024>(sa, sax, room);
    const float ma = sa * inv, max_ = sax * inv;
    for (uint32_t c = threadIdx.x; c < g.dim; c += 1024) {
      const float xh = (to_f32(x[c]) - mean) * rstd, d = to_f32(dy[c]);
      const float a = g.weight ? d * load_param<T>(g.weight, g.weight_f32, c) : d;
      dx[c] = from_f32<T>(rstd * (a - __builtin_fmaf(xh, max_, ma)));
    }
  }
}

// The partial sums of 64 columns, added in the order of the workgroups: 16 runs of them, then the runs.  (Bound by one read after
// another: with 16 at a time 10.5 -> 4.6 us for 512 parts of 768 columns.)
template <typename T>
__global__ __launch_bounds__(1024) void norm_grad_sum_kernel(const float *__restrict__ partial, uint32_t parts, uint32_t dim, void *dweight,
                                                             void *dbias, bool f32) {
  __shared__ float runs[16][64];
  const uint32_t lane = threadIdx.x % 64, run = threadIdx.x / 64;
  const uint64_t c = (uint64_t)blockIdx.x * 64 + lane;  // column of [2][dim]
  float sum = 0.0f;
  if (c < 2ull * dim) {
    const uint32_t end = (run + 1) * parts / 16;
    for (uint32_t p = run * parts / 16; p < end; p += 16) {  // 16 on their way at a time
      float v[16];
#pragma unroll
      for (uint32_t u = 0; u < 16; ++u) v[u] = p + u < end ? partial[(p + u) * 2ull * dim + c] : 0.0f;
#pragma unroll
      for (uint32_t u = 0; u < 16; ++u) sum += v[u];
    }
  }
  runs[run][lane] = sum;
  __syncthreads();
  if (run != 0 || c >= 2ull * dim) return;
  sum = 0.0f;
#pragma unroll
  for (int r = 0; r < 16; ++r) sum += runs[r][lane];
  void *out = c < dim ? dweight : dbias;
  if (out) store_param<T>(out, f32, c < dim ? c : c - dim, sum);
}

static uint32_t norm_parts(uint64_t n) { return (uint32_t)(n / 4 < 1 ? 1 : n / 4 < kNormParts ? n / 4 : kNormParts); }

// Launches one of the kernels above: the fewest lanes whose pieces hold the row.
template <typename T, int VEC, bool BACKWARD>
static void launch_norm_as(const NormArgs &g, hipStream_t st) {
  const auto run = [&](auto lanes) {
    constexpr int L = decltype(lanes)::value;
    constexpr int kGroups = kNormThreads<L> / L;
    const uint64_t want = (g.n + kGroups - 1) / kGroups;
    if constexpr (BACKWARD) {
      if (g.partial) {
        norm_grad_kernel<T, VEC, L, true><<<norm_parts(g.n), kNormThreads<L>, 0, st>>>(g);
      } else {
        norm_grad_kernel<T, VEC, L, false><<<(uint32_t)(want < kNormBlocks ? want : kNormBlocks), kNormThreads<L>, 0, st>>>(g);
      }
    } else {
      norm_kernel<T, VEC, L><<<(uint32_t)(want < kNormBlocks ? want : kNormBlocks), kNormThreads<L>, 0, st>>>(g);
    }
  };
  const uint32_t per_lane = kItems * VEC;
  if (g.dim <= 16 * per_lane)
    run(std::integral_constant<int, 16>());
  else if (g.dim <= 64 * per_lane)
    run(std::integral_constant<int, 64>());
  else if (g.dim <= 256 * per_lane)
    run(std::integral_constant<int, 256>());
  else if (g.dim <= 512 * per_lane)
    run(std::integral_constant<int, 512>());
  else if constexpr (BACKWARD)
    norm_grad_long_kernel<T><<<norm_parts(g.n), 1024, 0, st>>>(g);
  else
    norm_long_kernel<T><<<(uint32_t)(g.n < kNormBlocks ? g.n : kNormBlocks), 1024, 0, st>>>(g);
}

template <typename T, bool BACKWARD>
static void launch_norm(const NormArgs &g, hipStream_t st) {
  uint32_t b = piece_bytes(g.x, g.x_stride, g.dim, sizeof(T));
  const uint32_t by = piece_bytes(g.y, g.y_stride, g.dim, sizeof(T));
  if (by < b) b = by;
  if (BACKWARD) {
    const uint32_t bd = piece_bytes(g.dy, g.dy_stride, g.dim, sizeof(T));
    if (bd < b) b = bd;
  }
  if (b == 16)
    launch_norm_as<T, 16 / sizeof(T), BACKWARD>(g, st);
  else if (b == 8)
    launch_norm_as<T, 8 / sizeof(T), BACKWARD>(g, st);
  else
    launch_norm_as<T, 1, BACKWARD>(g, st);
}

template <bool BACKWARD>
static ann_status launch_norm_typed(uint32_t type, const NormArgs &g, hipStream_t st) {
  if (type == ANN_F32)
    launch_norm<float, BACKWARD>(g, st);
  else if (type == ANN_F16)
    launch_norm<f16_t, BACKWARD>(g, st);
  else
    launch_norm<bf16_t, BACKWARD>(g, st);
  ANN_HIP(hipGetLastError());
  return ANN_OK;
}

static ann_status check_norm(const char *what, uint64_t n, uint32_t dim, uint32_t type, uint32_t weight_type, bool params) {
  if (type > ANN_BF16) return fail(ANN_EINVAL, "%s: unknown type %u", what, type);
  if (params && weight_type != type && weight_type != ANN_F32)
    return fail(ANN_EINVAL, "%s: weights are of the rows' type or ANN_F32, not %u", what, weight_type);
  if (dim == 0) return fail(ANN_EINVAL, "%s: dim == 0", what);
  if (dim > ANN_MAX_NORM_DIM) return fail(ANN_ECAPACITY, "%s: dim = %u exceeds ANN_MAX_NORM_DIM = %u", what, dim, ANN_MAX_NORM_DIM);
  if (n >= (1ull << 40)) return fail(ANN_ECAPACITY, "%s: n = %llu", what, (unsigned long long)n);
  return ANN_OK;
}

}  // namespace ann

using namespace ann;

extern "C" ann_status ann_layer_norm(const void *x, uint64_t n, uint32_t dim, uint64_t x_stride, uint32_t type, const void *weight,
                                     const void *bias, uint32_t weight_type, float eps, void *y, uint64_t y_stride, float *mean, float *rstd,
                                     void *stream) {
  if (ann_status s = check_norm("ann_layer_norm", n, dim, type, weight_type, weight || bias)) return s;
  if (n == 0) return ANN_OK;
  if (!x || !y) return fail(ANN_EINVAL, "ann_layer_norm: NULL argument");
  if (x_stride < dim || y_stride < dim) return fail(ANN_EINVAL, "ann_layer_norm: a row stride is shorter than a row");
  if (!(eps >= 0.0f)) return fail(ANN_EINVAL, "ann_layer_norm: eps must not be negative");
  NormArgs g = {};
  g.x = x, g.weight = weight, g.bias = bias, g.y = y, g.mean = mean, g.rstd = rstd;
  g.n = n, g.x_stride = x_stride, g.y_stride = y_stride, g.dim = dim, g.eps = eps, g.weight_f32 = weight_type == ANN_F32;
  return launch_norm_typed<false>(type, g, (hipStream_t)stream);
}

extern "C" uint64_t ann_layer_norm_backward_workspace(uint64_t n, uint32_t dim) {
  return n == 0 ? 0 : (uint64_t)norm_parts(n) * 2 * dim * sizeof(float);
}

extern "C" ann_status ann_layer_norm_backward(const void *dy, uint64_t dy_stride, const void *x, uint64_t x_stride, uint64_t n, uint32_t dim,
                                              uint32_t type, const void *weight, uint32_t weight_type, const float *mean, const float *rstd,
                                              void *dx, uint64_t dx_stride, void *dweight, void *dbias, void *workspace,
                                              uint64_t workspace_bytes, void *stream) {
  const bool params = dweight || dbias;
  if (ann_status s = check_norm("ann_layer_norm_backward", n, dim, type, weight_type, weight || params)) return s;
  if (n && (!dy || !x || !mean || !rstd || !dx)) return fail(ANN_EINVAL, "ann_layer_norm_backward: NULL argument");
  if (n && (x_stride < dim || dy_stride < dim || dx_stride < dim))
    return fail(ANN_EINVAL, "ann_layer_norm_backward: a row stride is shorter than a row");
  const uint64_t need = params ? ann_layer_norm_backward_workspace(n, dim) : 0;
  if (need && !workspace) return fail(ANN_EINVAL, "ann_layer_norm_backward: workspace is NULL");
  if (workspace_bytes < need)
    return fail(ANN_EINVAL, "ann_layer_norm_backward: workspace of %llu bytes, %llu are needed", (unsigned long long)workspace_bytes,
                (unsigned long long)need);
  if ((uintptr_t)workspace % 4 && need) return fail(ANN_EINVAL, "ann_layer_norm_backward: workspace is not aligned to 4 bytes");
  const hipStream_t st = (hipStream_t)stream;
  NormArgs g = {};
  g.x = x, g.dy = dy, g.weight = weight, g.y = dx, g.mean = (float *)mean, g.rstd = (float *)rstd, g.partial = params ? (float *)workspace : nullptr;
  g.n = n, g.x_stride = x_stride, g.dy_stride = dy_stride, g.y_stride = dx_stride, g.dim = dim, g.weight_f32 = weight_type == ANN_F32;
  if (n)
    if (ann_status s = launch_norm_typed<true>(type, g, st)) return s;
  if (!params) return ANN_OK;
  const uint32_t parts = n ? norm_parts(n) : 0, grid = (2 * dim + 63) / 64;
  if (type == ANN_F16)
    norm_grad_sum_kernel<f16_t><<<grid, 1024, 0, st>>>(g.partial, parts, dim, dweight, dbias, g.weight_f32);
  else if (type == ANN_BF16)
    norm_grad_sum_kernel<bf16_t><<<grid, 1024, 0, st>>>(g.partial, parts, dim, dweight, dbias, g.weight_f32);
  else
    norm_grad_sum_kernel<float><<<grid, 1024, 0, st>>>(g.partial, parts, dim, dweight, dbias, true);
  ANN_HIP(hipGetLastError());
  return ANN_OK;
}
