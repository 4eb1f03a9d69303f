// What the operators on rows of a matrix share: sums and maxima over the lanes
// that hold a row, and 16-byte pieces of rows of any alignment and length.
#pragma once
#include "ann_internal.hpp"
#include "device_utils.hpp"
#include "scalar_types.hpp"

namespace ann {

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

// The sum and the maximum of one value over the LANES lanes that share a row.
template <int LANES>
__device__ __forceinline__ float row_sum(float v, float *room) {
  v = wave_sum(v, LANES < kWave ? LANES : kWave);
  if constexpr (LANES > kWave) {
    __syncthreads();  // the last row's has been read
    if (threadIdx.x % kWave == 0) room[threadIdx.x / kWave] = v;
    __syncthreads();
    v = 0.0f;
#pragma unroll
    for (int w = 0; w < LANES / kWave; ++w) v += room[w];
  }
  return v;
}

// Over aligned groups of `lanes` lanes, a power of two from 4 to 64.
__device__ __forceinline__ float lanes_max(float v, uint32_t lanes) {
  v = fmaxf(v, __int_as_float(dpp_i32<kDppQuadXor1>(__float_as_int(v))));
  v = fmaxf(v, __int_as_float(dpp_i32<kDppQuadXor2>(__float_as_int(v))));
  if (lanes >= 8) v = fmaxf(v, __int_as_float(dpp_i32<kDppRowHalfMirror>(__float_as_int(v))));
  if (lanes >= 16) v = fmaxf(v, __int_as_float(dpp_i32<kDppRowMirror>(__float_as_int(v))));
  if (lanes >= 32) {
    const LanePair p = lane_pair<true>(__float_as_uint(v));
    v = fmaxf(__uint_as_float(p.low), __uint_as_float(p.high));
  }
  if (lanes >= 64) {
    const LanePair p = lane_pair<false>(__float_as_uint(v));
    v = fmaxf(__uint_as_float(p.low), __uint_as_float(p.high));
  }
  return v;
}
template <int LANES>
__device__ __forceinline__ float row_max(float v, float *room) {
  v = lanes_max(v, LANES < kWave ? LANES : kWave);
  if constexpr (LANES > kWave) {
    __syncthreads();
    if (threadIdx.x % kWave == 0) room[threadIdx.x / kWave] = v;
    __syncthreads();
    v = room[0];
#pragma unroll
    for (int w = 1; w < LANES / kWave; ++w) v = fmaxf(v, room[w]);
  }
  return v;
}

// N elements from c on of a row of `columns`, with the alignment of one element: one access, or, at the row's end, one for
// each that there is; what lies behind it is read as zero and not written.
template <typename T, int N>
struct RowPiece {
  T v[N];
  __device__ __forceinline__ void load(const T *row, uint32_t c, uint32_t columns) {
    typedef Piece<T, N, sizeof(T)> P;
    if (c + N <= columns) {
      *(P *)v = *(const P *)(row + c);
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] = c + e < columns ? row[c + e] : (T)0.0f;
    }
  }
  __device__ __forceinline__ void store(T *row, uint32_t c, uint32_t columns) const {
    typedef Piece<T, N, sizeof(T)> P;
    if (c + N <= columns) {
      *(P *)(row + c) = *(const P *)v;
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (c + e < columns) row[c + e] = v[e];
    }
  }
};

}  // namespace ann
