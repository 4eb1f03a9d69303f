// Products of 128 x 128 tiles on the matrix cores, for the operators on rows'
// scores: C[m][n] += sum_k A[m][k] B[n][k], where either operand may lie in
// memory with k along the rows (kAlong) or down them (kAcross), with any stride,
// alignment and length.
//
// A workgroup of four wavefronts, 64 x 64 of the tile to a wavefront, two by two
// accumulators of the 32x32x16 instruction.  A slice of K is fetched into
// registers while the matrix cores work on the one before, then written to LDS.
// fp32 operands are split on the way into three bf16 planes (8 + 8 + 8 bits) and
// six of the nine products are taken; the three left out are below 2^-23 of the
// product together.  Operands that run down the rows are written to LDS as they
// come and transposed by ds_read_b64_tr_b16 on the way to the registers.
// 16-byte slots of a line of LDS are permuted with the line's number, so that
// lines read side by side hit all banks.
#pragma once
#include "ann_internal.hpp"
#include "device_utils.hpp"
#include "scalar_types.hpp"

namespace ann {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr int kTile = 128;  // lines of either operand to a tile
enum Order { kAlong, kAcross };

__device__ __forceinline__ f32x16 matrix_step(bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x16 matrix_step(f16x8 a, f16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }

// T: type in memory.  E: eight elements as the matrix instruction takes them.
template <typename T>
struct Operand16;
template <>
struct Operand16<bf16_t> {
  typedef bf16x8 E;
  static constexpr int kParts = 1, kSlice = 64;
};
template <>
struct Operand16<f16_t> {
  typedef f16x8 E;
  static constexpr int kParts = 1, kSlice = 64;
};
template <>
struct Operand16<float> {
  typedef bf16x8 E;
  static constexpr int kParts = 3, kSlice = 32;
};

// Lines line0 .. of a matrix whose element (line, k) is p[line * stride + k]
// (kAlong) or p[k * stride + line] (kAcross); lines and k below the given numbers exist.
template <typename T>
struct Lines {
  const T *p;
  uint64_t stride;
  uint32_t lines, depth;
  const float *bias = nullptr;  // kAcross: where bias[k] is -infinity, zeros are read
};

// Eight consecutive elements, `there` of which exist; the others are zero.
template <typename T>
struct Unit {
  T v[8];
};
template <typename T>
__device__ __forceinline__ void load_unit(Unit<T> &u, const T *p) {
  typedef Piece<T, 16 / sizeof(T), sizeof(T)> P;
  *(P *)u.v = *(const P *)p;
  if constexpr (sizeof(T) == 4) *(P *)(u.v + 4) = *(const P *)(p + 4);
}
template <typename T>
__device__ __forceinline__ void load_unit(Unit<T> &u, const T *p, int64_t there) {
  if (there >= 8) {
    load_unit(u, p);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) u.v[e] = e < there ? p[e] : (T)0.0f;
  }
}

__device__ __forceinline__ uint4 unit_part(const Unit<bf16_t> &u, int) { return __builtin_bit_cast(uint4, u); }
__device__ __forceinline__ uint4 unit_part(const Unit<f16_t> &u, int) { return __builtin_bit_cast(uint4, u); }
// Takes the part off: the remainders are exact.
__device__ __forceinline__ uint4 unit_part(Unit<float> &u, int) {
  bf16x8 h;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    h[e] = (bf16_t)u.v[e];
    // (an infinite element has no remainder: it stays in the first part alone)
    const float rest = __fsub_rn(u.v[e], (float)h[e]);
    u.v[e] = fabsf((float)h[e]) < INFINITY ? rest : 0.0f;
  }
  return __builtin_bit_cast(uint4, h);
}

template <typename T, Order ORDER>
struct TileSide {
  typedef Operand16<T> O;
  static constexpr int kUnits = kTile * O::kSlice / 8 / 256;  // to a lane
  static constexpr int kPlane = kTile * O::kSlice * 2;        // bytes
  static constexpr int kBytes = kPlane * O::kParts;
  Unit<T> u[kUnits];

  // Byte offset of 16-byte slot `slot` of line `line` of a plane.
  static __device__ __forceinline__ int slot_at(int line, int slot) {
    if constexpr (ORDER == kAcross)
      return line * (kTile * 2) + ((slot ^ ((line & 7) << 1)) << 4);  // lines are k: 256 bytes
    else if constexpr (O::kSlice == 64)
      return line * 128 + ((slot ^ (line & 7)) << 4);
    else
      return line * 64 + ((slot ^ ((line >> 1) & 3)) << 4);
  }
  // Where the lane's units lie from the tile's first element, in bytes.  Lines that do not exist are read as one that does: what
  // comes of them is not used.  (Offsets computed anew for every slice, with a test for each unit, took more
  // instructions than the product.)
  uint32_t from[kUnits];
  const char *base;
  bool direct;  // 32-bit offsets hold, and no unit ends behind the last line
  __device__ __forceinline__ void start(const Lines<T> &m, uint32_t line0) {
    const uint32_t last = m.lines - 1 - line0;  // (the tile has a line)
    base = (const char *)(m.p + (ORDER == kAlong ? line0 * m.stride : line0));
    direct = m.stride < (1u << 23) && (ORDER == kAlong || line0 + kTile <= m.lines || m.lines % 8 == 0);
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
      const uint32_t at = threadIdx.x + 256 * i;
      if constexpr (ORDER == kAlong) {
        uint32_t line = at / (O::kSlice / 8);
        line = line < last ? line : last;
        from[i] = (line * (uint32_t)m.stride + at % (O::kSlice / 8) * 8) * sizeof(T);
      } else {
        uint32_t line = at % (kTile / 8) * 8;
        line = line < last ? line : last / 8 * 8;
        from[i] = (at / (kTile / 8) * (uint32_t)m.stride + line) * sizeof(T);
      }
    }
  }
  __device__ __forceinline__ void fetch(const Lines<T> &m, uint32_t line0, uint32_t k0) {
    if (direct && k0 + O::kSlice <= m.depth && !(ORDER == kAcross && m.bias)) {
      const char *p = base + (ORDER == kAlong ? (uint64_t)k0 : k0 * m.stride) * sizeof(T);
#pragma unroll
      for (int i = 0; i < kUnits; ++i) load_unit(u[i], (const T *)(p + from[i]));
      return;
    }
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
      const uint32_t at = threadIdx.x + 256 * i;
      if constexpr (ORDER == kAlong) {
        const uint32_t line = line0 + at / (O::kSlice / 8), k = k0 + at % (O::kSlice / 8) * 8;
        load_unit(u[i], m.p + line * m.stride + k, line < m.lines ? (int64_t)m.depth - k : 0);
      } else {
        const uint32_t k = k0 + at / (kTile / 8), line = line0 + at % (kTile / 8) * 8;
        load_unit(u[i], m.p + k * m.stride + line, k < m.depth && !(m.bias && m.bias[k] == -INFINITY) ? (int64_t)m.lines - line : 0);
      }
    }
  }
  __device__ __forceinline__ void commit(char *lds) {
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
      const int at = (int)threadIdx.x + 256 * i;
      const int line = ORDER == kAlong ? at / (O::kSlice / 8) : at / (kTile / 8), slot = ORDER == kAlong ? at % (O::kSlice / 8) : at % (kTile / 8);
#pragma unroll
      for (int p = 0; p < O::kParts; ++p) *(uint4 *)(lds + p * kPlane + slot_at(line, slot)) = unit_part(u[i], p);
    }
  }
  // What the lane brings to the matrix instruction: eight k of one line (k = 16 kk + 8 (lane / 32) .., line = 32 block + lane % 32).
  static __device__ __forceinline__ typename O::E fragment(const char *lds, int part, int block, int kk) {
    const int lane = lane_id();
    lds += part * kPlane;
    if constexpr (ORDER == kAlong) {
      return *(const typename O::E *)(lds + slot_at(block * 32 + lane % 32, kk * 2 + lane / 32));
    } else {
      // 16 lanes read 4 k of 16 lines, 4 lines of one k to a lane, and get 4 k of one line each
      union {
        s16x4 half[2];
        typename O::E e;
      } f;
      const int line = block * 32 + lane / 16 % 2 * 16 + lane % 4 * 4;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int k = kk * 16 + lane / 32 * 8 + h * 4 + lane % 16 / 4;
        f.half[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (__attribute__((address_space(3))) s16x4 *)(lds + slot_at(k, line / 8) + line % 8 * 2));
      }
      return f.e;
    }
  }
};

template <typename T, Order OA, Order OB>
constexpr int kTileBytes = TileSide<T, OA>::kBytes + TileSide<T, OB>::kBytes;

template <int M, int N>
__device__ __forceinline__ void clear(f32x16 (&acc)[M][N]) {
#pragma unroll
  for (int i = 0; i < M; ++i)
#pragma unroll
    for (int j = 0; j < N; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;
}

// acc[i][j]: 32 x 32 block (m block 2 (wave / 2) + i, n block 2 (wave % 2) + j).  Lane l
// holds column n = l % 32 and rows m = 8 (r / 4) + 4 (l / 32) + r % 4, r = 0 .. 15.
// All 256 lanes take part; lds: kTileBytes bytes, free when the call begins after a barrier.
// APART (fp32): the five smaller products of parts are summed by themselves, so that the sum rounds once per 16 k and not six times.
template <typename T, Order OA, Order OB, bool APART = false>
__device__ __forceinline__ void tile_product(f32x16 (&acc)[2][2], const Lines<T> &A, uint32_t m0, const Lines<T> &B, uint32_t n0,
                                             uint32_t k_begin, uint32_t k_end, char *lds) {
  typedef Operand16<T> O;
  typedef TileSide<T, OA> SA;
  typedef TileSide<T, OB> SB;
  char *lb = lds + SA::kBytes;
  SA a;
  SB b;
  const int mw = (int)(threadIdx.x / kWave) / 2 * 2, nw = (int)(threadIdx.x / kWave) % 2 * 2;
  f32x16 low[2][2];
  if constexpr (APART) clear(low);
  a.start(A, m0), b.start(B, n0);
  if (k_begin < k_end) a.fetch(A, m0, k_begin), b.fetch(B, n0, k_begin);
  for (uint32_t k = k_begin; k < k_end; k += O::kSlice) {
    __syncthreads();  // the slice before has been read
    a.commit(lds);
    b.commit(lb);
    __syncthreads();
    if (k + O::kSlice < k_end) a.fetch(A, m0, k + O::kSlice), b.fetch(B, n0, k + O::kSlice);
#pragma unroll
    for (int kk = 0; kk < O::kSlice / 16; ++kk) {
      typename O::E fa[O::kParts][2], fb[O::kParts][2];
#pragma unroll
      for (int p = 0; p < O::kParts; ++p)
#pragma unroll
        for (int i = 0; i < 2; ++i) fa[p][i] = SA::fragment(lds, p, mw + i, kk), fb[p][i] = SB::fragment(lb, p, nw + i, kk);
#pragma unroll
      for (int sum = O::kParts - 1; sum >= 0; --sum)  // the smallest products first
#pragma unroll
        for (int p = 0; p <= sum; ++p)
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              f32x16 &to = APART && sum != 0 ? low[i][j] : acc[i][j];
              to = matrix_step(fa[p][i], fb[sum - p][j], to);
            }
    }
  }
  if constexpr (APART) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[i][j][r] += low[i][j][r];
  }
}

// Products of 256 x 128 tiles of 16-bit elements for operands whose addresses and strides are multiples of 16 bytes: 128 x 64 of
// the tile to a wavefront (a 64 x 64 share reads LDS for twice the cycles that the matrix cores take).  Slices of 32 k go from
// memory straight into one of three buffers of LDS, two slices ahead (one ahead, the product waited for memory: each slice has lines that
// the L2 does not hold), and fragments are read beside the products of the ones before.  Two such workgroups share a
// compute unit: the end of one's tile lies beside the other's product.  870 TFLOP/s of fp16 with long rows (a library's large product:
// 1,190); LDS is busy for three cycles where the matrix cores are for two (writes from memory take it for 16 cycles per KiB).
constexpr int kWideM = 256, kWideN = 128, kWideSlice = 32;
constexpr int kWideBuffer = (kWideM + kWideN) * kWideSlice * 2;

inline bool wide_operand(const void *p, uint64_t stride) { return (uintptr_t)p % 16 == 0 && stride % 8 == 0 && stride < (1u << 23); }

// kAlong: the depth is a multiple of 32; kAcross: the number of lines is one of 8, and lines of k behind the last are read as the last
// (the other operand is zero there).
template <typename T, Order ORDER, int LINES>
struct WideSide {
  typedef typename Operand16<T>::E E;
  static constexpr int kUnits = LINES * kWideSlice / 8 / 256;
  static constexpr int kBytes = LINES * kWideSlice * 2;
  static constexpr int kSlots = ORDER == kAlong ? kWideSlice / 8 : LINES / 8;  // of 16 bytes to a line of LDS
  // A unit's place in LDS is its number; the slot in memory that it holds is permuted with its line.
  static __device__ __forceinline__ int permuted(int line, int slot) { return ORDER == kAlong ? slot ^ ((line >> 1) & 3) : slot ^ ((line & 7) << 1); }
  const char *base;
  uint32_t from[kUnits];
  __device__ __forceinline__ void start(const Lines<T> &m, uint32_t line0) {
    const uint32_t last = m.lines - 1 - line0;  // (lines that do not exist are read as one that does)
    base = (const char *)(m.p + (ORDER == kAlong ? line0 * m.stride : line0));
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
      const int at = (int)threadIdx.x + 256 * i, along = at / kSlots, slot = permuted(along, at % kSlots);
      if constexpr (ORDER == kAlong) {
        const uint32_t line = (uint32_t)along < last ? (uint32_t)along : last;
        from[i] = (line * (uint32_t)m.stride + slot * 8) * sizeof(T);
      } else {
        const uint32_t line = (uint32_t)slot * 8 < last ? (uint32_t)slot * 8 : last / 8 * 8;
        from[i] = (along * (uint32_t)m.stride + line) * sizeof(T);
      }
    }
  }
  __device__ __forceinline__ void fetch(const Lines<T> &m, uint32_t k0, char *lds) {
    typedef const __attribute__((address_space(1))) void *From;
    typedef __attribute__((address_space(3))) void *To;
    const char *p = base + (ORDER == kAlong ? (uint64_t)k0 : k0 * m.stride) * sizeof(T);
    if (ORDER == kAcross && k0 + kWideSlice > m.depth) {
#pragma unroll
      for (int i = 0; i < kUnits; ++i) {
        const uint32_t k = k0 + (threadIdx.x + 256 * i) / kSlots;
        if (k >= m.depth) from[i] -= (k - (m.depth - 1)) * (uint32_t)m.stride * sizeof(T);  // (the last slice: from is not used again)
      }
    }
    char *to = lds + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave) * (kWave * 16);
#pragma unroll
    for (int i = 0; i < kUnits; ++i) __builtin_amdgcn_global_load_lds((From)(p + from[i]), (To)(to + i * 4096), 16, 0, 0);
  }
  // Eight k of one line (k = 16 kk + 8 (lane / 32) .., line = 32 block + lane % 32).
  static __device__ __forceinline__ E fragment(const char *lds, int block, int kk) {
    const int lane = lane_id();
    if constexpr (ORDER == kAlong) {
      return *(const E *)(lds + (block * 32 + lane % 32) * (kSlots * 16) + (permuted(lane % 32, kk * 2 + lane / 32) << 4));
    } else {
      union {
        s16x4 half[2];
        E e;
      } f;
      const int line = block * 32 + lane / 16 % 2 * 16 + lane % 4 * 4;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int k = kk * 16 + lane / 32 * 8 + h * 4 + lane % 16 / 4;
        f.half[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (__attribute__((address_space(3))) s16x4 *)(lds + k * (kSlots * 16) + (permuted(k, line / 8) << 4) + line % 8 * 2));
      }
      return f.e;
    }
  }
};

// Waits until at most `on_their_way` of the lane's reads into LDS (0 or a slice's) are outstanding and its own reads of LDS are done, then for
// the other wavefronts.
template <int ON_THEIR_WAY>
__device__ __forceinline__ void wide_barrier() {
  static_assert(ON_THEIR_WAY < 16, "");
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0x0070 | ON_THEIR_WAY);  // vmcnt(ON_THEIR_WAY) lgkmcnt(0)
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// acc[i][j]: 32 x 32 block (m block 4 (wave / 2) + i, n block 2 (wave % 2) + j).  k_begin and the depths: see WideSide.  The three
// buffers of kWideBuffer bytes are variables of their own (so that the compiler can tell reads of one from what is on its way into
// another) and free when the call begins after a barrier.  All 256 lanes take part.  SOME: wavefronts for which `mine` is false add nothing (what A holds of
// their lines is not looked at).
template <typename T, Order OA, Order OB, bool SOME = false>
__device__ __forceinline__ void wide_product(f32x16 (&acc)[4][2], const Lines<T> &A, uint32_t m0, const Lines<T> &B, uint32_t n0, uint32_t k_begin,
                                             uint32_t k_end, char *lds0, char *lds1, char *lds2, bool mine = true) {
  typedef WideSide<T, OA, kWideM> SA;
  typedef WideSide<T, OB, kWideN> SB;
  typedef typename Operand16<T>::E E;
  constexpr int kInFlight = SA::kUnits + SB::kUnits;
  if (k_begin >= k_end) return;
  SA a;
  SB b;
  a.start(A, m0), b.start(B, n0);
  const int mw = (int)(threadIdx.x / kWave) / 2 * 4, nw = (int)(threadIdx.x / kWave) % 2 * 2;
  const uint32_t slices = (k_end - k_begin + kWideSlice - 1) / kWideSlice;
  const auto fetch = [&](uint32_t s, char *to) { a.fetch(A, k_begin + s * kWideSlice, to), b.fetch(B, k_begin + s * kWideSlice, to + SA::kBytes); };
  E fa[2][4], fb[2][2];  // of the first and the second 16 k of a slice
  const auto read = [&](const char *at, int kk) {
#pragma unroll
    for (int i = 0; i < 4; ++i) fa[kk][i] = SA::fragment(at, mw + i, kk);
#pragma unroll
    for (int j = 0; j < 2; ++j) fb[kk][j] = SB::fragment(at + SA::kBytes, nw + j, kk);
  };
  const auto multiply = [&](int kk) {
    if (SOME && !mine) return;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) acc[i][j] = matrix_step(fa[kk][i], fb[kk][j], acc[i][j]);
  };
  __syncthreads();  // the last readers of the buffers are done
  fetch(0, lds0);
  if (slices > 1) fetch(1, lds1);
  if (slices > 2) fetch(2, lds2);
  if (slices > 2)
    wide_barrier<2 * kInFlight>();
  else
    wide_barrier<0>();
  read(lds0, 0);
  // Slice s, whose first fragments have been read.
  const auto step = [&](uint32_t s, char *now, const char *next) {
    __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0): the first fragments, before more are asked for that need not be waited for
    read(now, 1);
    __builtin_amdgcn_sched_barrier(0);
    multiply(0);
    // slice s + 1 is there, and slice s is in all wavefronts' registers
    if (s + 2 < slices)
      wide_barrier<kInFlight>();
    else
      wide_barrier<0>();
    read(next, 0);  // (behind the last slice: whatever is there, not used)
    if (s + 3 < slices) fetch(s + 3, now);
    __builtin_amdgcn_sched_barrier(0);
    multiply(1);
    __builtin_amdgcn_sched_barrier(0);
  };
  uint32_t s = 0;
  for (; s + 3 <= slices; s += 3) {
    step(s, lds0, lds1);
    step(s + 1, lds1, lds2);
    step(s + 2, lds2, lds0);
  }
  if (s < slices) step(s, lds0, lds1);
  if (s + 1 < slices) step(s + 1, lds1, lds2);
}

// Row of a 32 x 32 block that register r of the lane's half holds.
__device__ __forceinline__ int block_row(int r) { return r / 4 * 8 + lane_id() / 32 * 4 + r % 4; }

}  // namespace ann
