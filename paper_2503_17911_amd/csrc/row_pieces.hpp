// What the operators on rows of a matrix share: sums and maxima over the lanes
// that hold a row, and 16-byte pieces of rows of any alignment and length.
#pragma once
#include <type_traits>

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

// Elements of type T in words of 32 bits, as they lie in memory.  (Pieces are kept as words: as elements, what two branches load is taken apart
// and put together again, at twice the registers and the time.)
template <typename T>
__device__ __forceinline__ float word_f32(uint32_t w, int half) {
  if constexpr (sizeof(T) == 4)
    return __uint_as_float(w);
  else if constexpr (std::is_same<T, bf16_t>::value)
    return __uint_as_float(half ? w & 0xFFFF0000u : w << 16);
  else
    return to_f32(__builtin_bit_cast(T, (uint16_t)(half ? w >> 16 : w)));
}
template <typename T>
__device__ __forceinline__ uint32_t f32_word(float a, float b) {
  return (uint32_t)__builtin_bit_cast(uint16_t, from_f32<T>(a)) | (uint32_t)__builtin_bit_cast(uint16_t, from_f32<T>(b)) << 16;
}

// N words at any address that ALIGN divides.
template <int N, int ALIGN>
struct __attribute__((packed, aligned(ALIGN), may_alias)) Words {
  uint32_t v[N];
};

// How a row ends: with a whole piece; within one, which is read as the row's last N elements and shifted into place (reads stay in
// flight side by side; rows shorter than a piece element by element); within one that is read element by element
// (no element is read by two lanes: for rows in place that several wavefronts share).
enum RowEnd { kWholePieces, kShifted, kByElement };

// N elements from c on of a row of `columns`, with the alignment of one element; what lies behind the row is read as zero and not written.
template <typename T, int N, RowEnd END = kByElement>
struct RowPiece {
  static constexpr int kPer = 4 / (int)sizeof(T), kWords = N / kPer;  // elements to a word
  typedef Words<kWords, sizeof(T)> P;
  typedef typename std::conditional<sizeof(T) == 4, uint32_t, uint16_t>::type U __attribute__((may_alias));
  uint32_t w[kWords];
  __device__ __forceinline__ float get(int e) const { return word_f32<T>(w[e / kPer], e % kPer); }
  __device__ __forceinline__ void set(const float (&v)[N]) {
#pragma unroll
    for (int k = 0; k < kWords; ++k) {
      if constexpr (kPer == 1)
        w[k] = __float_as_uint(v[k]);
      else
        w[k] = f32_word<T>(v[2 * k], v[2 * k + 1]);
    }
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int k = 0; k < kWords; ++k) w[k] = 0;
  }
  __device__ __forceinline__ void read(const T *at) {
    const P p = *(const P *)at;
#pragma unroll
    for (int k = 0; k < kWords; ++k) w[k] = p.v[k];
  }
  __device__ __forceinline__ void load(const T *row, uint32_t c, uint32_t columns) {
    if (END == kShifted && columns >= N) {
      const uint32_t from = c + N <= columns ? c : columns - N, by = c - from;  // by elements, N and more: nothing is left
      read(row + from);
#pragma unroll
      for (int step = 1; step <= kWords; step *= 2)
#pragma unroll
        for (int k = 0; k < kWords; ++k) w[k] = by / kPer & step ? (k + step < kWords ? w[k + step < kWords ? k + step : 0] : 0) : w[k];
      if constexpr (kPer == 2) {
#pragma unroll
        for (int k = 0; k < kWords; ++k) w[k] = by & 1 ? __builtin_amdgcn_alignbit(k + 1 < kWords ? w[k + 1 < kWords ? k + 1 : 0] : 0, w[k], 16) : w[k];
      }
      if (by >= N) clear();
    } else if (END == kWholePieces ? c < columns : c + N <= columns) {
      read(row + c);
    } else {
      clear();
      if (END != kWholePieces && c < columns) {
#pragma unroll
        for (int e = 0; e < N; ++e)
          if (c + e < columns) w[e / kPer] |= (uint32_t)((const U *)row)[c + e] << (e % kPer * 16);
      }
    }
  }
  // Past the caches.
  __device__ __forceinline__ void store_past(T *row, uint32_t c, uint32_t columns) const {
    typedef uint32_t Vector __attribute__((ext_vector_type(4)));
    typedef Vector Unaligned __attribute__((aligned(2), may_alias));
    if (kWords == 4 && (END == kWholePieces ? c < columns : c + N <= columns)) {
      const Vector v = {w[0], w[1 % kWords], w[2 % kWords], w[3 % kWords]};
      __builtin_nontemporal_store(v, (Unaligned *)(row + c));
    } else {
      store(row, c, columns);
    }
  }
  __device__ __forceinline__ void store(T *row, uint32_t c, uint32_t columns) const {
    if (END == kWholePieces ? c < columns : c + N <= columns) {
      P p;
#pragma unroll
      for (int k = 0; k < kWords; ++k) p.v[k] = w[k];
      *(P *)(row + c) = p;
    } else if (END != kWholePieces && c < columns) {
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (c + e < columns) ((U *)row)[c + e] = (U)(w[e / kPer] >> (e % kPer * 16));
    }
  }
};

}  // namespace ann
