// Shared device building blocks of the operators on feature rows: 16-byte
// pieces of a row at any element alignment, and sums over groups of lanes.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "spconv_rows.h"

namespace spc {

// Element types of the rows: float, and bf16 as raw 16 bits.
typedef uint16_t bf16_t;

template <typename T> struct Row;
template <> struct Row<float> {
  static constexpr int VEC = 4;                    // elements per 16-byte piece
  __device__ static float get(float v) { return v; }
  __device__ static float put(float v) { return v; }
};
template <> struct Row<bf16_t> {
  static constexpr int VEC = 8;
  __device__ static float get(bf16_t v) { return __uint_as_float(static_cast<uint32_t>(v) << 16); }
  __device__ static bf16_t put(float v) {
    return __builtin_bit_cast(bf16_t, static_cast<__bf16>(v));   // nearest even, NaN quiet
  }
};

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

// A 16-byte piece from / to memory aligned to the element only (gfx950 takes
// such accesses in one instruction; where the address happens to be aligned
// they cost nothing extra).
template <typename T> __device__ __forceinline__ u32x4_t load_piece(const T* p) {
  u32x4_t v;
  __builtin_memcpy(&v, p, 16);
  return v;
}
template <typename T> __device__ __forceinline__ void store_piece(T* p, u32x4_t v) {
  __builtin_memcpy(p, &v, 16);
}

// The same past the caches' replacement order: for an output far larger than the
// L2 cache, which would otherwise push out what is still to be read.
template <typename T> __device__ __forceinline__ void store_piece_past(T* p, u32x4_t v) {
  typedef uint32_t any_t __attribute__((ext_vector_type(4), aligned(2)));
  __builtin_nontemporal_store(v, reinterpret_cast<any_t*>(p));
}

__device__ __forceinline__ void unpack(u32x4_t u, float (&v)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(u[i]);
}
__device__ __forceinline__ void unpack(u32x4_t u, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(u[i] << 16);
    v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ u32x4_t pack(const float (&v)[4]) {
  u32x4_t u;
#pragma unroll
  for (int i = 0; i < 4; ++i) u[i] = __float_as_uint(v[i]);
  return u;
}
// Two values rounded to bf16 by one instruction.
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  typedef float f2 __attribute__((ext_vector_type(2)));
  typedef __bf16 b2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f2{a, b}), b2));
}
__device__ __forceinline__ u32x4_t pack(const float (&v)[8]) {
  u32x4_t u;
#pragma unroll
  for (int i = 0; i < 4; ++i) u[i] = pack2(v[2 * i], v[2 * i + 1]);
  return u;
}

// Elements [c, c + VEC) of a row of C elements at p, those past the end 0.
// TAIL false: C is a multiple of VEC (or the caller knows the piece is whole).
template <typename T, bool TAIL>
__device__ __forceinline__ void load_row(const T* p, int64_t c, int64_t C,
                                         float (&v)[Row<T>::VEC]) {
  constexpr int VEC = Row<T>::VEC;
  if (!TAIL || c + VEC <= C) {
    unpack(load_piece(p + c), v);
  } else {
#pragma unroll
    for (int i = 0; i < VEC; ++i) v[i] = c + i < C ? Row<T>::get(p[c + i]) : 0.0f;
  }
}
template <typename T, bool TAIL>
__device__ __forceinline__ void store_row(T* p, int64_t c, int64_t C,
                                          const float (&v)[Row<T>::VEC]) {
  constexpr int VEC = Row<T>::VEC;
  if (!TAIL || c + VEC <= C) {
    store_piece(p + c, pack(v));
  } else {
#pragma unroll
    for (int i = 0; i < VEC; ++i)
      if (c + i < C) p[c + i] = Row<T>::put(v[i]);
  }
}
// VEC fp32 elements (a parameter of the columns) with the same guard.
template <int VEC, bool TAIL>
__device__ __forceinline__ void load_f32(const float* p, int64_t c, int64_t C, float (&v)[VEC]) {
  if (!TAIL || c + VEC <= C) {
#pragma unroll
    for (int q = 0; q < VEC; q += 4) {
      const u32x4_t u = load_piece(p + c + q);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[q + i] = __uint_as_float(u[i]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < VEC; ++i) v[i] = c + i < C ? p[c + i] : 0.0f;
  }
}

// The value of the lane at the other end of a butterfly step of 1, 2, 4 or 8
// lanes (4 and 8 by mirroring, which pairs lanes whose smaller groups already
// hold equal values), on the vector ALU's data-parallel primitives.
template <int STEP> __device__ __forceinline__ uint32_t lane_other(uint32_t v) {
  constexpr int ctrl = STEP == 1 ? 0xB1 : STEP == 2 ? 0x4E : STEP == 4 ? 0x141 : 0x140;
  return static_cast<uint32_t>(
      __builtin_amdgcn_update_dpp(0, static_cast<int>(v), ctrl, 0xf, 0xf, true));
}

// op over the aligned group of LPR lanes this lane is in (LPR a power of two
// up to 64); every lane of the group ends with the same bits.
template <int LPR, typename Op> __device__ __forceinline__ float group_reduce(float v, Op op) {
  if constexpr (LPR > 1) v = op(v, __uint_as_float(lane_other<1>(__float_as_uint(v))));
  if constexpr (LPR > 2) v = op(v, __uint_as_float(lane_other<2>(__float_as_uint(v))));
  if constexpr (LPR > 4) v = op(v, __uint_as_float(lane_other<4>(__float_as_uint(v))));
  if constexpr (LPR > 8) v = op(v, __uint_as_float(lane_other<8>(__float_as_uint(v))));
  if constexpr (LPR > 16) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false,
                                                    false);
    v = op(__uint_as_float(r[0]), __uint_as_float(r[1]));
  }
  if constexpr (LPR > 32) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false,
                                                    false);
    v = op(__uint_as_float(r[0]), __uint_as_float(r[1]));
  }
  return v;
}
template <int LPR> __device__ __forceinline__ float group_sum(float v) {
  return group_reduce<LPR>(v, [](float a, float b) { return a + b; });
}

// The same over a workgroup of 256 lanes through LDS (4 floats each in turn at
// s[0..3] and s[4..7]: `turn` alternates, so one barrier a call is enough).
__device__ __forceinline__ float block_sum(float v, float* s, int turn) {
  v = group_sum<64>(v);
  float* t = s + 4 * (turn & 1);
  if ((threadIdx.x & 63) == 0) t[threadIdx.x >> 6] = v;
  __syncthreads();
  return (t[0] + t[1]) + (t[2] + t[3]);
}

// ---------------------------------------------------------------------------
// Host side: argument checks, and what the entry points call.
// ---------------------------------------------------------------------------
inline bool aligned_to(const void* p, size_t a) {
  return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0;
}
inline size_t elem_bytes(int dt) { return dt == SPCONV_BF16 ? 2 : 4; }
inline bool dtype_ok(int dt) { return dt == SPCONV_F32 || dt == SPCONV_BF16; }
// A pointer to `count` elements: there when any are, and aligned.
inline bool ptr_ok(const void* p, int64_t count, size_t bytes) {
  return (p || count == 0) && aligned_to(p, bytes);
}
inline bool rows_ok(int64_t n) { return n >= 0 && n < 0x80000000ll; }
// A launch holds fewer than 2^32 threads.
inline bool grid_fits(int64_t blocks, int threads) { return blocks < (1ll << 32) / threads; }
inline int launched() { return hipGetLastError() == hipSuccess ? SPCONV_OK : SPCONV_EHIP; }

}  // namespace spc
