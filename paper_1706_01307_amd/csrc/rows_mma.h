// Shared device building blocks of the products of feature rows: operand tiles in LDS
// for the matrix cores, the ring of stages that feeds them, and finished tiles' ways out.
#pragma once

#include "rows.h"

namespace spc {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));

// Consecutive workgroups go to the 8 dies in turn, each with an L2 of its own:
// tiles are dealt so that a die has a contiguous run of them (the column tiles
// of one row tile, and the row tiles of one group, share their operands).
__device__ __forceinline__ int64_t die_order(int64_t b, int64_t total) {
  const int64_t per = total / 8, rem = total % 8, die = b % 8;
  return die * per + (die < rem ? die : rem) + b / 8;
}

// The matrix-core step per type.  Operand fragments are [32 rows][KS] with the
// reduction contiguous per lane; D = first x second^T has the first operand's
// rows at 8 (i / 4) + 4 (lane / 32) + i % 4 and the second's at lane % 32.
template <typename T> struct Mma;
template <> struct Mma<bf16_t> {
  static constexpr int KS = 16;                    // reduction of a fragment
  typedef bf16x8 Frag;
  __device__ static f32x16 mma(Frag a, Frag b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  }
};
template <> struct Mma<float> {
  static constexpr int KS = 8;
  typedef f32x4_t Frag;
  __device__ static f32x16 mma(Frag a, Frag b, f32x16 c) {
#pragma unroll
    for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[i], b[i], c, 0, 0, 0);
    return c;
  }
};

// Staged tiles in LDS, in 16-byte pieces; a stage is KB bytes of the reduction,
// BK elements.
//
// RTile: R rows of KB bytes.  A fragment read takes one piece column of 16 rows
// per cycle, so pieces are permuted by the row: 16 rows then cover the 64 banks
// once.
template <typename T, int KB> constexpr int kBK = KB / static_cast<int>(sizeof(T));

// A lane's place in a tile, for reads at constant distances from it: hidden from
// the compiler, which would otherwise keep every sum with a tile's address and
// step in a register of its own.
__device__ __forceinline__ int lane_place(int byte) {
  asm volatile("" : "+v"(byte));
  return byte;
}
template <typename V> __device__ __forceinline__ V lds_at(const u32x4_t* t, int byte) {
  return *reinterpret_cast<const V*>(reinterpret_cast<const char*>(t) + byte);
}

template <typename T, int R, int KB> struct RTile {
  static constexpr int PR = KB / 16;               // pieces per row
  static constexpr int PIECES = R * PR, STEPS = PR / 2;
  __device__ static int at(int row, int piece) {
    return row * PR + (piece ^ (KB == 128 ? (row >> 1) & 7 : (row >> 2) & 3));
  }
  // fragments of rows r0 + 32 b .. + 31, the reduction's step s (pieces 2 s, 2 s + 1)
  struct Reader {
    int place[STEPS];
    __device__ Reader(int r0, int lane) {
#pragma unroll
      for (int s = 0; s < STEPS; ++s)
        place[s] = lane_place(at(r0 + (lane & 31), 2 * s + (lane >> 5)) * 16);
    }
    __device__ typename Mma<T>::Frag operator()(const u32x4_t* t, int b, int s) const {
      return lds_at<typename Mma<T>::Frag>(t, place[s] + b * 32 * KB);
    }
  };
};
// KTile: BK rows of the reduction of W columns each; fragments are read across
// the rows.  bf16: LDS reads that transpose 4 x 16 blocks; 64-byte spans of four
// rows must lie in different banks.  fp32: one element a lane; the two halves of
// a wave read rows 4 apart.
template <typename T, int W, int KB> struct KTile {
  static constexpr int VEC = Row<T>::VEC, PR = W / VEC;   // pieces per row
  static constexpr int PIECES = kBK<T, KB> * PR;
  __device__ static int at(int k, int piece) {
    if constexpr (sizeof(T) == 2) {
      const int x = W >= 128 ? (k & 3) << 2 : W == 64 ? ((k >> 1) & 1) << 2 : 0;
      return k * PR + (piece ^ x);
    } else {
      return k * PR + (piece ^ (W >= 64 ? ((k >> 2) & 1) << 3 : 0));
    }
  }
  // fragments of columns c0 + B b .. + 31 (b < NB), the reduction's step s
  template <int B, int NB> struct Reader {
    int place[NB];
    __device__ Reader(int c0, int lane) {
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        if constexpr (sizeof(T) == 2) {
          // lanes 16 q + j ask for row 8 (q / 2) + j / 4, columns 16 (q % 2) + 4 (j % 4) .. + 3,
          // and receive column lane % 32 of rows 8 (lane / 32) .. + 3
          const int j = lane & 15, q = lane >> 4;
          const int row = 8 * (q >> 1) + (j >> 2), col = c0 + B * b + 16 * (q & 1) + 4 * (j & 3);
          place[b] = lane_place(at(row, col >> 3) * 16 + (col & 7) * 2);
        } else {
          const int col = c0 + B * b + (lane & 31);
          place[b] = lane_place(at(4 * (lane >> 5), col >> 2) * 16 + (col & 3) * 4);
        }
      }
    }
    __device__ typename Mma<T>::Frag operator()(const u32x4_t* t, int b, int s) const {
      const int at = place[b] + s * Mma<T>::KS * PR * 16;
      if constexpr (sizeof(T) == 2) {
        typedef __attribute__((address_space(3))) s16x4 lds_s4;
        const char* p = reinterpret_cast<const char*>(t) + at;
        lds_s4* lo = (lds_s4*)(const_cast<char*>(p));
        lds_s4* hi = (lds_s4*)(const_cast<char*>(p) + 4 * PR * 16);
        const s16x4 u = __builtin_amdgcn_ds_read_tr16_b64_v4i16(lo);
        const s16x4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16(hi);
        const s16x8 r = {u[0], u[1], u[2], u[3], v[0], v[1], v[2], v[3]};
        return __builtin_bit_cast(bf16x8, r);
      } else {
        f32x4_t f;
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = lds_at<float>(t, at + i * PR * 16);
        return f;
      }
    }
  };
};

// What a lane reads where there is nothing to read: a load that always happens
// needs no branch, and its value no test.
__device__ const u32x4_t g_zeros = {0u, 0u, 0u, 0u};

// A piece of a row: `left` elements of it remain (<= 0: none, zeros).
// WHOLE: remaining counts are multiples of a piece.
template <typename T, bool WHOLE>
__device__ __forceinline__ u32x4_t load_left(const T* p, int64_t left) {
  constexpr int VEC = Row<T>::VEC;
  if constexpr (WHOLE) {
    return load_piece(left > 0 ? p : reinterpret_cast<const T*>(&g_zeros));
  } else {
    u32x4_t v = {0u, 0u, 0u, 0u};
    if (left >= VEC) {
      v = load_piece(p);
    } else if (left > 0) {
      T e[VEC];
#pragma unroll
      for (int i = 0; i < VEC; ++i) e[i] = i < left ? p[i] : T(0);
      __builtin_memcpy(&v, e, 16);
    }
    return v;
  }
}
template <typename TO, bool PAST = false>
__device__ __forceinline__ void store_left(TO* p, u32x4_t v, int64_t left) {
  constexpr int VO = Row<TO>::VEC;
  if (left >= VO) {
    if (PAST) store_piece_past(p, v); else store_piece(p, v);
  } else {
    TO e[VO];
    __builtin_memcpy(e, &v, 16);
#pragma unroll
    for (int i = 0; i < VO; ++i)
      if (i < left) p[i] = e[i];
  }
}

// 16 bytes a lane from global memory (16-byte aligned) straight to LDS: lane i's
// go to l + 16 i, l the same for the whole wave.  They are read behind a
// stage_barrier().
__device__ __forceinline__ void load_to_lds(const void* g, u32x4_t* l) {
  typedef __attribute__((address_space(3))) void lds_void;
  typedef __attribute__((address_space(1))) const void global_void;
  __builtin_amdgcn_global_load_lds((global_void*)g, (lds_void*)l, 16, 0, 0);
}
// The barrier of a ring of stages: every wave waits for its own loads, all but the
// LATER last ones (those of later stages), and for its LDS reads.  Behind it this
// stage is in LDS and the buffer of the one before is free.  (__syncthreads would
// wait for all loads.)
template <int LATER> __device__ __forceinline__ void stage_barrier() {
  asm volatile("" ::: "memory");
  // vmcnt(LATER), lgkmcnt(0)
  __builtin_amdgcn_s_waitcnt(0x0070 | (LATER & 15) | (LATER >> 4) << 14);
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// Finished rows in LDS as rows of CW columns; pieces are permuted by the row, so
// that the 32 rows of a write and the rows of a read lie in different banks.
template <typename TO, int CW> __device__ __forceinline__ int out_at(int r, int piece) {
  constexpr int PR = CW / Row<TO>::VEC;
  return r * PR + (piece ^ (r & (PR - 1)));
}

// A stage's products of a wave: FM x FN blocks.  (Fragments read a step ahead into
// a second set of registers, with or without an order given to the scheduler,
// were no faster: the two waves a SIMD has take turns.)
template <typename T, int KB, int FM, int FN, typename LoadA, typename LoadB>
__device__ __forceinline__ void multiply_stage(f32x16 (&acc)[FN][FM], LoadA la, LoadB lb) {
  typedef Mma<T> M;
#pragma unroll
  for (int q = 0; q < kBK<T, KB> / M::KS; ++q) {
    typename M::Frag fa[FM], fb[FN];
#pragma unroll
    for (int m = 0; m < FM; ++m) fa[m] = la(m, q);
#pragma unroll
    for (int n = 0; n < FN; ++n) fb[n] = lb(n, q);
#pragma unroll
    for (int n = 0; n < FN; ++n)
#pragma unroll
      for (int m = 0; m < FM; ++m) acc[n][m] = M::mma(fb[n], fa[m], acc[n][m]);
    __builtin_amdgcn_sched_barrier(0);
  }
}

// Where a wave's column block n starts: the blocks of a tile's waves lie side by
// side, so that a part of the finished tile is of adjacent columns.
template <int WC> __device__ __forceinline__ int col_of(int wcol, int n) {
  return 32 * (wcol + WC * n);
}

__device__ __forceinline__ void put4(float* d, const float (&v)[4]) {
  *reinterpret_cast<float4*>(d) = make_float4(v[0], v[1], v[2], v[3]);
}
__device__ __forceinline__ void put4(bf16_t* d, const float (&v)[4]) {
  *reinterpret_cast<uint2*>(d) = make_uint2(pack2(v[0], v[1]), pack2(v[2], v[3]));
}

// 4 x 4 exchange among the four lanes of a quad: lane i's v[j] becomes lane j's
// v[i].
__device__ __forceinline__ void quad_transpose(uint32_t (&v)[4]) {
  const bool odd = threadIdx.x & 1, high = threadIdx.x & 2;
#pragma unroll
  for (int j = 0; j < 4; j += 2) {
    const uint32_t r = lane_other<1>(odd ? v[j] : v[j + 1]);
    if (odd) v[j] = r; else v[j + 1] = r;
  }
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const uint32_t r = lane_other<2>(high ? v[j] : v[j + 2]);
    if (high) v[j] = r; else v[j + 2] = r;
  }
}

// v of lane i + D within 16 lanes (rotating), D = 4 or 8
template <int D> __device__ __forceinline__ float row_rotate(float v) {
  return __uint_as_float(static_cast<uint32_t>(__builtin_amdgcn_update_dpp(
      0, static_cast<int>(__float_as_uint(v)), 0x120 | D, 0xf, 0xf, true)));
}
// A lane's part of the column sums of a fragment (the same column in both halves
// of the wave, other rows).
__device__ __forceinline__ float frag_sum(float s, bf16x8 f) {
#pragma unroll
  for (int i = 0; i < 8; ++i) s += static_cast<float>(f[i]);
  return s;
}
__device__ __forceinline__ float frag_sum(float s, f32x4_t f) {
#pragma unroll
  for (int i = 0; i < 4; ++i) s += f[i];
  return s;
}

// Whole aligned 16-byte pieces in rows of C elements from p.
template <typename T> bool whole_rows(const void* p, int64_t C) {
  return C % Row<T>::VEC == 0 && aligned_to(p, 16);
}

}  // namespace
}  // namespace spc
