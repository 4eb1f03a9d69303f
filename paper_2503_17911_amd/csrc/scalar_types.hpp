// Element types of the operators on hidden states (ann_type) and 16-byte
// pieces of rows of them.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ann.h"

namespace ann {

typedef __bf16 bf16_t;
typedef _Float16 f16_t;

constexpr uint32_t type_bytes(uint32_t type) { return type == ANN_F32 ? 4u : 2u; }

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(f16_t v) { return (float)v; }
__device__ __forceinline__ float to_f32(bf16_t v) { return __uint_as_float((uint32_t)__builtin_bit_cast(uint16_t, v) << 16); }

// One rounding to nearest, ties to even (bf16: v_cvt_pk_bf16_f32).
template <typename T>
__device__ __forceinline__ T from_f32(float v) {
  return (T)v;
}

// N elements that are read or written by one instruction where N * sizeof(T)
// is 16 bytes (ALIGN: the alignment that the caller promises).
template <typename T, int N, int ALIGN = N * (int)sizeof(T)>
struct alignas(ALIGN) Piece {
  T v[N];
};

// Loads and stores an fp32 or T value of a parameter vector (weights come in either).
template <typename T>
__device__ __forceinline__ float load_param(const void *p, bool f32, uint64_t i) {
  return f32 ? ((const float *)p)[i] : to_f32(((const T *)p)[i]);
}
template <typename T>
__device__ __forceinline__ void store_param(void *p, bool f32, uint64_t i, float v) {
  if (f32)
    ((float *)p)[i] = v;
  else
    ((T *)p)[i] = from_f32<T>(v);
}

// How many bytes of an array of rows may be read or written at a time: the
// largest power of two up to 16 that divides its address and its row stride,
// if `columns` is a whole number of such pieces.
inline uint32_t piece_bytes(const void *p, uint64_t stride, uint32_t columns, uint32_t elem) {
  uint32_t b = 16;
  while (b > elem && (((uintptr_t)p | (stride * elem)) % b != 0 || ((uint64_t)columns * elem) % b != 0)) b >>= 1;
  return b;
}

}  // namespace ann
