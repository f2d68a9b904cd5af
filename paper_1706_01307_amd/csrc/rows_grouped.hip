// Products of ragged groups of rows, each group with its own weights, and their
// gradients, on the matrix cores.
//
// Which rows a workgroup has is found on the device: the groups' row tiles are
// numbered in order, and each wave finds the tile's group by a running sum over
// the offsets, 64 groups at a time.  No host knows the group sizes.
#include "rows.h"

namespace spc {
namespace {

constexpr int kThreads = 256;

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));

// A run of positions of one group: [begin, end), of the group's tile `index`.
struct Tile {
  int group;                   // E: the positions behind the last group; -1: none
  int64_t begin, end;          // the tile's positions
  int index;                   // which of the group's tiles
};

// Tile t of the groups cut into tiles of BM positions, the positions behind
// the last group as group E (WITH_TAIL).  Every wave of the workgroup calls it
// and gets the same answer.  Offsets are moved into [0, m]; a group never
// reaches beyond them.
template <bool WITH_TAIL>
__device__ __forceinline__ Tile find_tile(const int32_t* __restrict__ offsets, int E, int64_t m,
                                          int64_t BM, int64_t t) {
  const int lane = threadIdx.x & 63;
  const int groups = E + (WITH_TAIL ? 1 : 0);
  int64_t before = 0;
  for (int e0 = 0; e0 < groups; e0 += 64) {
    const int e = e0 + lane;
    int64_t a = 0, b = 0;
    if (e < groups) {
      a = offsets[e];
      b = e < E ? offsets[e + 1] : m;
      a = a < 0 ? 0 : a > m ? m : a;
      b = b < 0 ? 0 : b > m ? m : b;
    }
    const int64_t len = b > a ? b - a : 0;
    const int tiles = static_cast<int>((len + BM - 1) / BM);
    int sum = tiles;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const int o = __shfl_up(sum, d, 64);
      if (lane >= d) sum += o;
    }
    const uint64_t hit = __ballot(before + sum > t);
    if (hit) {
      const int src = __ffsll(static_cast<unsigned long long>(hit)) - 1;
      Tile r;
      r.group = e0 + src;
      r.index = static_cast<int>(t - before) - (__shfl(sum, src, 64) - __shfl(tiles, src, 64));
      const int64_t ga = __shfl(a, src, 64), gb = __shfl(b, src, 64);
      r.begin = ga + static_cast<int64_t>(r.index) * BM;
      r.end = r.begin + BM < gb ? r.begin + BM : gb;
      return r;
    }
    before += __shfl(sum, 63, 64);
  }
  return Tile{-1, 0, 0, 0};
}

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
  __device__ static Frag ones() {
    Frag f;
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = static_cast<__bf16>(1.0f);
    return f;
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
  __device__ static Frag ones() { return Frag{1.0f, 1.0f, 1.0f, 1.0f}; }
};

// Staged tiles in LDS, in 16-byte pieces: a stage is 128 bytes of the reduction
// (BK elements), so that a row's load is a whole cache line (with 64 bytes the
// address unit took 55 cycles an instruction instead of 17 and bounded both
// kernels).
//
// RTile: R rows of BK elements.  A fragment read takes one piece column of 16
// rows per cycle, so pieces are permuted by the row's bits 1 to 3: 16 rows then
// cover the 64 banks once.
template <typename T> constexpr int kBK = 128 / static_cast<int>(sizeof(T));
template <typename T, int R> struct RTile {
  static constexpr int PIECES = R * 8, BYTES = R * 128;
  __device__ static int at(int row, int piece) { return row * 8 + (piece ^ ((row >> 1) & 7)); }
  // rows r0..r0+31, reduction from piece 2 s
  __device__ static typename Mma<T>::Frag frag(const u32x4_t* t, int r0, int s, int lane) {
    return __builtin_bit_cast(typename Mma<T>::Frag, t[at(r0 + (lane & 31), 2 * s + (lane >> 5))]);
  }
};
// KTile: BK rows of the reduction of W columns each; fragments are read across
// the rows.  bf16: LDS reads that transpose 4 x 16 blocks; 64-byte spans of four
// rows must lie in different banks.  fp32: one element a lane; the two halves of
// a wave read rows 4 apart.
template <typename T, int W> struct KTile {
  static constexpr int VEC = Row<T>::VEC, PR = W / VEC;   // pieces per row
  static constexpr int PIECES = kBK<T> * PR, BYTES = PIECES * 16;
  __device__ static int at(int k, int piece) {
    if constexpr (sizeof(T) == 2) {
      const int x = W >= 128 ? (k & 3) << 2 : W == 64 ? ((k >> 1) & 1) << 2 : 0;
      return k * PR + (piece ^ x);
    } else {
      return k * PR + (piece ^ (W >= 64 ? ((k >> 2) & 1) << 3 : 0));
    }
  }
  // columns c0..c0+31, reduction from row KS * s
  __device__ static typename Mma<T>::Frag frag(const u32x4_t* t, int c0, int s, int lane) {
    if constexpr (sizeof(T) == 2) {
      // lanes 16 q + j ask for row 8 (q / 2) + j / 4, columns 16 (q % 2) + 4 (j % 4) .. + 3,
      // and receive column lane % 32 of rows 8 (lane / 32) .. + 3
      const int j = lane & 15, q = lane >> 4;
      const int row = 16 * s + 8 * (q >> 1) + (j >> 2), col = c0 + 16 * (q & 1) + 4 * (j & 3);
      typedef __attribute__((address_space(3))) s16x4 lds_s4;
      const uint16_t* b = reinterpret_cast<const uint16_t*>(t);
      lds_s4* lo = (lds_s4*)(const_cast<uint16_t*>(b) + at(row, col >> 3) * 8 + (col & 7));
      lds_s4* hi = (lds_s4*)(const_cast<uint16_t*>(b) + at(row + 4, col >> 3) * 8 + (col & 7));
      const s16x4 u = __builtin_amdgcn_ds_read_tr16_b64_v4i16(lo);
      const s16x4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16(hi);
      const s16x8 r = {u[0], u[1], u[2], u[3], v[0], v[1], v[2], v[3]};
      return __builtin_bit_cast(bf16x8, r);
    } else {
      const float* b = reinterpret_cast<const float*>(t);
      const int col = c0 + (lane & 31);
      f32x4_t f;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        f[i] = b[at(8 * s + 4 * (lane >> 5) + i, col >> 2) * 4 + (col & 3)];
      return f;
    }
  }
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
template <typename TO>
__device__ __forceinline__ void store_left(TO* p, u32x4_t v, int64_t left) {
  constexpr int VO = Row<TO>::VEC;
  if (left >= VO) {
    store_piece(p, v);
  } else {
    TO e[VO];
    __builtin_memcpy(e, &v, 16);
#pragma unroll
    for (int i = 0; i < VO; ++i)
      if (i < left) p[i] = e[i];
  }
}

// A wave's FM blocks of 32 x 32 of one column block go to LDS, rounded, as rows
// of CW columns (the first operand's rows are the columns: a lane has 4 adjacent
// ones of one row in every four registers).  Pieces are permuted by the row, so
// that the 32 rows of a write and the rows of a read lie in different banks.
template <typename TO, int CW> __device__ __forceinline__ int out_at(int r, int piece) {
  constexpr int PR = CW / Row<TO>::VEC;
  return r * PR + (piece ^ (r & (PR - 1)));
}
template <typename TO, int CW, int FM>
__device__ __forceinline__ void block_to_lds(u32x4_t* s, const f32x16 (&acc)[FM], int r0, int c0,
                                             const float (&bias)[16], int relu) {
  constexpr int VO = Row<TO>::VEC;
  const int lane = threadIdx.x & 63, h = lane >> 5;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int c = c0 + 8 * q + 4 * h;
#pragma unroll
    for (int m = 0; m < FM; ++m) {
      const int r = r0 + 32 * m + (lane & 31);
      TO v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float z = acc[m][4 * q + i] + bias[4 * q + i];
        if (relu && z < 0.0f) z = 0.0f;
        v[i] = Row<TO>::put(z);
      }
      TO* d = reinterpret_cast<TO*>(s + out_at<TO, CW>(r, c / VO)) + c % VO;
      __builtin_memcpy(__builtin_assume_aligned(d, 4 * sizeof(TO)), v, sizeof v);
    }
  }
}

struct GroupedArgs {
  const void* x;               // [n_x][red]
  int64_t n_x;
  const void* w;
  const int32_t* offsets;
  const int32_t* rows;         // NULL: position j reads row j
  const float* bias;
  const void* mask;
  int relu;
  void* y;                     // [m][cols]
  int64_t m;
  int E, red, cols;            // reduction, output columns
  int strip;                   // column tiles a workgroup takes
  hipStream_t st;
};

// Rows x weights: BT false: w[e] is [red][cols] (the forward), BT true: w[e] is
// [cols][red] (the input gradient).  A workgroup takes BM positions of a group
// and `strip` column tiles of BN one after the other, four waves in 2 x 2.  Its
// stages (128 bytes of the reduction of one column tile) run on across the
// column tiles: the next kDepth stages' pieces are on their way into registers
// while one, in LDS, is multiplied; two LDS buffers, one barrier a stage.  A
// finished tile leaves through the buffer that is free then, as whole rows (in
// 32-byte parts of rows, stored from the registers, the forward wrote 1.8 times
// its bytes to memory).
template <typename T, typename TO, bool BT, int BM, int BN, bool WHOLE>
__global__ __launch_bounds__(kThreads, 2) void k_grouped(GroupedArgs a) {
  typedef Mma<T> M;
  typedef RTile<T, BM> TA;
  typedef RTile<T, BN> TBr;
  typedef KTile<T, BN> TBk;
  constexpr int VEC = Row<T>::VEC, BK = kBK<T>, STEPS = BK / M::KS, kDepth = 2;
  constexpr int FM = BM / 64, FN = BN / 64;
  constexpr int PA = TA::PIECES / kThreads;
  constexpr int PB = TBk::PIECES / kThreads;       // (as many as TBr's)
  constexpr int kStage = TA::BYTES + TBk::BYTES;
  __shared__ __attribute__((aligned(16))) unsigned char s_buf[2 * kStage];
  const T* const x = static_cast<const T*>(a.x);
  TO* const y = static_cast<TO*>(a.y);
  const int ncol = (a.cols + BN - 1) / BN, nstrip = (ncol + a.strip - 1) / a.strip;
  const int64_t id = die_order(blockIdx.x, gridDim.x);
  const Tile t = find_tile<true>(a.offsets, a.E, a.m, BM, id / nstrip);
  if (t.group < 0) return;
  const int tile0 = static_cast<int>(id % nstrip) * a.strip;
  const int ntile = ncol - tile0 < a.strip ? ncol - tile0 : a.strip;
  const int nrow = static_cast<int>(t.end - t.begin);
  if (t.group == a.E) {                            // behind the last group
    const int64_t c0 = static_cast<int64_t>(tile0) * BN;
    const int64_t c1 = c0 + static_cast<int64_t>(ntile) * BN;
    const int64_t end = c1 < a.cols ? c1 : a.cols;
    for (int r = 0; r < nrow; ++r)
      for (int64_t c = c0 + threadIdx.x; c < end; c += kThreads)
        y[(t.begin + r) * a.cols + c] = Row<TO>::put(0.0f);
    return;
  }
  const T* const w = static_cast<const T*>(a.w) + static_cast<int64_t>(t.group) * a.red * a.cols;

  // what this lane stages of the rows: rows (threadIdx.x >> 3) + 32 i, the
  // piece threadIdx.x & 7 of each stage.  A row that is not there is read as
  // zeros, at one place all along (step 0).
  const int ka = (threadIdx.x & 7) * VEC;
  const T* pa[PA];
  int step[PA];
#pragma unroll
  for (int i = 0; i < PA; ++i) {
    const int r = (threadIdx.x >> 3) + 32 * i;
    int64_t src = -1;
    if (r < nrow) {
      src = a.rows ? a.rows[t.begin + r] : t.begin + r;
      if (src >= a.n_x) src = -1;
    }
    step[i] = src >= 0 ? BK : 0;
    pa[i] = src >= 0 ? x + src * a.red + ka : reinterpret_cast<const T*>(&g_zeros);
  }
  const int nk = (a.red + BK - 1) / BK, nstage = nk * ntile;
  // and of the weights, from the stage's own place; columns past the last one
  // are read as the last ones (nothing of them is stored)
  uint32_t pb[PB];
  auto weights_at = [&](int n0) {
#pragma unroll
    for (int i = 0; i < PB; ++i) {
      if constexpr (BT) {
        const int n = (threadIdx.x >> 3) + 32 * i;
        pb[i] = static_cast<uint32_t>(n0 + n < a.cols ? n : 0) * a.red + ka;
      } else {
        const int p = threadIdx.x + kThreads * i, n = p % TBk::PR * VEC;
        pb[i] = static_cast<uint32_t>(p / TBk::PR) * a.cols + (n0 + n < a.cols ? n : 0);
      }
    }
  };
  u32x4_t ra[kDepth][PA], rb[kDepth][PB];
  int rk = 0, rn = tile0 * BN;                     // the next stage to request
  weights_at(rn);
  auto request = [&](int d) {
    if (WHOLE && rk + BK <= a.red) {
#pragma unroll
      for (int i = 0; i < PA; ++i) {
        ra[d][i] = load_piece(pa[i]);
        pa[i] += step[i];
      }
      const T* ws = BT ? w + static_cast<int64_t>(rn) * a.red + rk
                       : w + static_cast<int64_t>(rk) * a.cols + rn;
#pragma unroll
      for (int i = 0; i < PB; ++i) rb[d][i] = load_piece(ws + pb[i]);
    } else {
      // the end of the reduction, or pieces that may be cut
#pragma unroll
      for (int i = 0; i < PA; ++i) {
        ra[d][i] = load_left<T, WHOLE>(pa[i], step[i] ? a.red - rk - ka : 0);
        pa[i] += step[i];
      }
#pragma unroll
      for (int i = 0; i < PB; ++i) {
        if constexpr (BT) {
          const int n = rn + (threadIdx.x >> 3) + 32 * i;
          rb[d][i] = load_left<T, WHOLE>(w + static_cast<int64_t>(n) * a.red + rk + ka,
                                         n < a.cols ? a.red - rk - ka : 0);
        } else {
          const int p = threadIdx.x + kThreads * i;
          const int k = rk + p / TBk::PR, n = rn + p % TBk::PR * VEC;
          rb[d][i] = load_left<T, WHOLE>(w + static_cast<int64_t>(k) * a.cols + n,
                                         k < a.red ? a.cols - n : 0);
        }
      }
    }
    rk += BK;
    if (rk >= a.red) {                             // on to the next column tile
      rk = 0;
      rn += BN;
#pragma unroll
      for (int i = 0; i < PA; ++i) pa[i] -= static_cast<int64_t>(nk) * step[i];
      weights_at(rn);
    }
  };
  auto put = [&](int d, int buf) {
    u32x4_t* sa = reinterpret_cast<u32x4_t*>(s_buf + buf * kStage);
    u32x4_t* sb = reinterpret_cast<u32x4_t*>(s_buf + buf * kStage + TA::BYTES);
#pragma unroll
    for (int i = 0; i < PA; ++i)
      sa[TA::at((threadIdx.x >> 3) + 32 * i, threadIdx.x & 7)] = ra[d][i];
#pragma unroll
    for (int i = 0; i < PB; ++i) {
      if constexpr (BT) {
        sb[TBr::at((threadIdx.x >> 3) + 32 * i, threadIdx.x & 7)] = rb[d][i];
      } else {
        const int p = threadIdx.x + kThreads * i;
        sb[TBk::at(p / TBk::PR, p % TBk::PR)] = rb[d][i];
      }
    }
  };

  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int wr = (wave >> 1) * (BM / 2), wc = (wave & 1) * (BN / 2);
  f32x16 acc[FN][FM];
  auto clear = [&] {
#pragma unroll
    for (int n = 0; n < FN; ++n)
#pragma unroll
      for (int m = 0; m < FM; ++m)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[n][m][i] = 0.0f;
  };
  // The tile's columns leave in parts of CW, FN / PARTS column blocks of each
  // wave column, through one buffer.
  constexpr int VO = Row<TO>::VEC;
  constexpr int PARTS = BM * BN * static_cast<int>(sizeof(TO)) > kStage ? 2 : 1;
  static_assert(FN % PARTS == 0 && BM * BN / PARTS * static_cast<int>(sizeof(TO)) <= kStage,
                "a part of the tile fits a buffer");
  constexpr int CW = BN / PARTS, HW = CW / 2;      // columns of a part; of a wave column's half
  auto finish = [&](int n0, int buf) {
    u32x4_t* so = reinterpret_cast<u32x4_t*>(s_buf + buf * kStage);
    const float* bias = a.bias ? a.bias + static_cast<int64_t>(t.group) * a.cols : nullptr;
#pragma unroll
    for (int part = 0; part < PARTS; ++part) {
      if (part) __syncthreads();
#pragma unroll
      for (int f = 0; f < FN / PARTS; ++f) {
        const int n = part * (FN / PARTS) + f;
        float b[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) b[i] = 0.0f;
        if (bias) {
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int c = n0 + wc + 32 * n + 8 * (i / 4) + 4 * (lane >> 5) + i % 4;
            b[i] = bias[c < a.cols ? c : 0];
          }
        }
        block_to_lds<TO, CW, FM>(so, acc[n], wr, (wave & 1) * HW + 32 * f, b, a.relu);
      }
      __syncthreads();
      for (int p = threadIdx.x; p < BM * CW / VO; p += kThreads) {
        const int r = p / (CW / VO), piece = p % (CW / VO), c = piece * VO;
        const int col = n0 + (c / HW) * (BN / 2) + part * HW + c % HW, left = a.cols - col;
        if (r >= nrow || left <= 0) continue;
        const int64_t at = (t.begin + r) * a.cols + col;
        u32x4_t u = so[out_at<TO, CW>(r, piece)];
        if (a.mask) {
          float v[VO], g[VO];
          unpack(u, v);
          unpack(load_left<TO, false>(static_cast<const TO*>(a.mask) + at, left), g);
#pragma unroll
          for (int i = 0; i < VO; ++i) v[i] = g[i] <= 0.0f ? 0.0f : v[i];
          u = pack(v);
        }
        store_left(y + at, u, left);
      }
    }
    __syncthreads();
  };

#pragma unroll
  for (int d = 0; d < kDepth; ++d)
    if (d < nstage) request(d);
  clear();
  int k = 0, n0 = tile0 * BN;
  for (int s0 = 0; s0 < nstage; s0 += kDepth) {
#pragma unroll
    for (int d = 0; d < kDepth; ++d) {
      if (s0 + d >= nstage) break;
      const int buf = d & 1;                       // (kDepth is even)
      put(d, buf);
      if (s0 + d + kDepth < nstage) request(d);
      __syncthreads();
      const u32x4_t* sa = reinterpret_cast<const u32x4_t*>(s_buf + buf * kStage);
      const u32x4_t* sb = reinterpret_cast<const u32x4_t*>(s_buf + buf * kStage + TA::BYTES);
#pragma unroll
      for (int s = 0; s < STEPS; ++s) {
        typename M::Frag fa[FM], fb[FN];
#pragma unroll
        for (int m = 0; m < FM; ++m) fa[m] = TA::frag(sa, wr + 32 * m, s, lane);
#pragma unroll
        for (int n = 0; n < FN; ++n) {
          if constexpr (BT) fb[n] = TBr::frag(sb, wc + 32 * n, s, lane);
          else fb[n] = TBk::frag(sb, wc + 32 * n, s, lane);
        }
#pragma unroll
        for (int n = 0; n < FN; ++n)
#pragma unroll
          for (int m = 0; m < FM; ++m) acc[n][m] = M::mma(fb[n], fa[m], acc[n][m]);
      }
      if (++k == nk) {
        finish(n0, buf ^ 1);
        clear();
        k = 0;
        n0 += BN;
      }
    }
  }
}

// Weight gradient of a BC x BN tile of one group, over a chunk of its
// positions: dw[c][n] = sum_j x[row j][c] dy[j][n].  Both operands are staged
// with the positions as the reduction's rows.  Chunk `id` leaves its sums as
// part[id] (one chunk per group: dw[group] itself).  The column-tile-0
// workgroups also sum dy, as the product of ones with it.
struct WeightArgs {
  const void* x;
  int64_t n_x;
  const void* dy;
  const int32_t* offsets;
  const int32_t* rows;
  float *dw, *db;              // where chunk / group g's sums go
  int64_t m, chunk;            // chunk = 0: a group is one chunk
  int E, C_in, C_out;
  hipStream_t st;
};

template <typename T, int BC, int BN, bool WHOLE>
__global__ __launch_bounds__(kThreads, 2) void k_grouped_dw(WeightArgs a) {
  typedef Mma<T> M;
  typedef KTile<T, BC> TX;
  typedef KTile<T, BN> TY;
  constexpr int VEC = Row<T>::VEC, BK = kBK<T>, STEPS = BK / M::KS, kDepth = 2;
  constexpr int FC = BC / 64, FN = BN / 64;
  constexpr int PX = TX::PIECES / kThreads, PY = TY::PIECES / kThreads;
  constexpr int kStage = TX::BYTES + TY::BYTES;
  __shared__ __attribute__((aligned(16))) unsigned char s_buf[2 * kStage];
  const T *const x = static_cast<const T*>(a.x), *const dy = static_cast<const T*>(a.dy);
  const int64_t nc = (a.C_in + BC - 1) / BC, nn = (a.C_out + BN - 1) / BN;
  const int64_t id = die_order(blockIdx.x, gridDim.x);
  const int64_t job = id / (nc * nn), c0 = id / nn % nc * BC, n0 = id % nn * BN;
  Tile t;
  if (a.chunk) {
    t = find_tile<false>(a.offsets, a.E, a.m, a.chunk, job);
    if (t.group < 0) return;
  } else {
    int64_t b = a.offsets[job], e = a.offsets[job + 1];
    b = b < 0 ? 0 : b > a.m ? a.m : b;
    e = e < b ? b : e > a.m ? a.m : e;
    t = Tile{static_cast<int>(job), b, e, 0};
  }
  // The row numbers of kThreads positions at a time, three such runs in LDS: the
  // one being requested, the next one, and the one a slower wave may still read.
  __shared__ int32_t s_row[3][kThreads];
  constexpr int RUN = kThreads / BK;               // stages of a run
  auto row_of = [&](int64_t j) {
    return j >= t.end ? -1 : a.rows ? a.rows[j] : static_cast<int32_t>(j);
  };
  int64_t rj = t.begin;                            // the next stage to request
  int rq = 0, run = 0;                             // its place in its run, its run (mod 3)
  s_row[0][threadIdx.x] = row_of(rj + threadIdx.x);
  int32_t row_next = row_of(rj + kThreads + threadIdx.x);
  __syncthreads();
  u32x4_t rx[kDepth][PX], ry[kDepth][PY];
  uint32_t py[PY];
#pragma unroll
  for (int i = 0; i < PY; ++i) {
    const int p = threadIdx.x + kThreads * i, n = p % TY::PR * VEC;
    py[i] = static_cast<uint32_t>(p / TY::PR) * a.C_out + (n0 + n < a.C_out ? n : 0);
  }
  auto request = [&](int d) {
#pragma unroll
    for (int i = 0; i < PX; ++i) {
      const int p = threadIdx.x + kThreads * i;
      const int32_t row = s_row[run][rq * BK + p / TX::PR];
      const int64_t c = c0 + p % TX::PR * VEC;
      const bool ok = row >= 0 && row < a.n_x;
      rx[d][i] = load_left<T, WHOLE>(x + static_cast<int64_t>(row) * a.C_in + c,
                                     ok ? a.C_in - c : 0);
    }
    if (WHOLE && rj + BK <= t.end) {
      // (columns past the last one are read as others: nothing of them is stored)
      const T* ys = dy + rj * a.C_out + n0;
#pragma unroll
      for (int i = 0; i < PY; ++i) ry[d][i] = load_piece(ys + py[i]);
    } else {
#pragma unroll
      for (int i = 0; i < PY; ++i) {
        const int p = threadIdx.x + kThreads * i;
        const int64_t j = rj + p / TY::PR, n = n0 + p % TY::PR * VEC;
        ry[d][i] = load_left<T, WHOLE>(dy + j * a.C_out + n, j < t.end ? a.C_out - n : 0);
      }
    }
    if (rq == 0) {
      // (read from the next stage but RUN - 1 on, with barriers between)
      const int to = run == 2 ? 0 : run + 1;
      s_row[to][threadIdx.x] = row_next;
      row_next = row_of(rj + 2 * kThreads + threadIdx.x);
    }
    rj += BK;
    if (++rq == RUN) {
      rq = 0;
      run = run == 2 ? 0 : run + 1;
    }
  };
  auto put = [&](int d, int buf) {
    u32x4_t* sx = reinterpret_cast<u32x4_t*>(s_buf + buf * kStage);
    u32x4_t* sy = reinterpret_cast<u32x4_t*>(s_buf + buf * kStage + TX::BYTES);
#pragma unroll
    for (int i = 0; i < PX; ++i) {
      const int p = threadIdx.x + kThreads * i;
      sx[TX::at(p / TX::PR, p % TX::PR)] = rx[d][i];
    }
#pragma unroll
    for (int i = 0; i < PY; ++i) {
      const int p = threadIdx.x + kThreads * i;
      sy[TY::at(p / TY::PR, p % TY::PR)] = ry[d][i];
    }
  };
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int wr = (wave >> 1) * (BC / 2), wc = (wave & 1) * (BN / 2);
  const bool bias = a.db && c0 == 0 && wr == 0;    // (uniform over the wave)
  f32x16 acc[FN][FC], accb[FN];
#pragma unroll
  for (int n = 0; n < FN; ++n)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      accb[n][i] = 0.0f;
#pragma unroll
      for (int m = 0; m < FC; ++m) acc[n][m][i] = 0.0f;
    }
  const int64_t nk = (t.end - t.begin + BK - 1) / BK;
#pragma unroll
  for (int d = 0; d < kDepth; ++d)
    if (d < nk) request(d);
  for (int64_t k0 = 0; k0 < nk; k0 += kDepth) {
#pragma unroll
    for (int d = 0; d < kDepth; ++d) {
      if (k0 + d >= nk) break;
      const int buf = d & 1;
      put(d, buf);
      if (k0 + d + kDepth < nk) request(d);
      __syncthreads();
      const u32x4_t* sx = reinterpret_cast<const u32x4_t*>(s_buf + buf * kStage);
      const u32x4_t* sy = reinterpret_cast<const u32x4_t*>(s_buf + buf * kStage + TX::BYTES);
#pragma unroll
      for (int s = 0; s < STEPS; ++s) {
        typename M::Frag fx[FC], fy[FN];
#pragma unroll
        for (int m = 0; m < FC; ++m) fx[m] = TX::frag(sx, wr + 32 * m, s, lane);
#pragma unroll
        for (int n = 0; n < FN; ++n) fy[n] = TY::frag(sy, wc + 32 * n, s, lane);
#pragma unroll
        for (int n = 0; n < FN; ++n)
#pragma unroll
          for (int m = 0; m < FC; ++m) acc[n][m] = M::mma(fy[n], fx[m], acc[n][m]);
        if (bias) {
#pragma unroll
          for (int n = 0; n < FN; ++n) accb[n] = M::mma(fy[n], M::ones(), accb[n]);
        }
      }
    }
  }
  // every column of the product with ones holds the same sums
  if (bias && (lane & 31) == 0) {
#pragma unroll
    for (int n = 0; n < FN; ++n)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int64_t col = n0 + wc + 32 * n + 8 * (i / 4) + 4 * (lane >> 5) + i % 4;
        if (col < a.C_out) a.db[job * a.C_out + col] = accb[n][i];
      }
  }
  float* out = a.dw + job * a.C_in * a.C_out;
#pragma unroll
  for (int n = 0; n < FN; ++n)
#pragma unroll
    for (int m = 0; m < FC; ++m) {
      const int64_t r = c0 + wr + 32 * m + (lane & 31);
      if (r >= a.C_in) continue;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int64_t c = n0 + wc + 32 * n + 8 * q + 4 * (lane >> 5);
        float v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = acc[n][m][4 * q + i];
        if (c < a.C_out) store_left(out + r * a.C_out + c, pack(v), a.C_out - c);
      }
    }
}

// The chunks' sums of a group, in ascending order: dw | db of one group as a
// row of C_in * C_out + C_out values, four a lane.
__global__ __launch_bounds__(kThreads) void k_grouped_dw_sum(
    const float* __restrict__ part, const float* __restrict__ part_db,
    const int32_t* __restrict__ offsets, int E, int64_t m, int64_t chunk, int64_t per, int C_out,
    float* __restrict__ dw, float* __restrict__ db) {
  __shared__ int64_t s_first, s_count;
  const int e = blockIdx.y;
  if (threadIdx.x < 64) {
    // chunks before group e, and its own
    int64_t before = 0, own = 0;
    for (int g = threadIdx.x; g <= e; g += 64) {
      int64_t b = offsets[g], f = offsets[g + 1];
      b = b < 0 ? 0 : b > m ? m : b;
      f = f < b ? b : f > m ? m : f;
      const int64_t c = (f - b + chunk - 1) / chunk;
      if (g < e) before += c; else own = c;
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      before += __shfl_xor(before, d, 64);
      own += __shfl_xor(own, d, 64);
    }
    if (threadIdx.x == 0) {
      s_first = before;
      s_count = own;
    }
  }
  __syncthreads();
  const int64_t first = s_first, count = s_count;
  const int64_t i = (static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x) * 4;
  if (i < per) {
    f32x4_t a = {0.0f, 0.0f, 0.0f, 0.0f};
    if (i + 4 <= per) {
#pragma unroll 4
      for (int64_t c = 0; c < count; ++c)
        a += __builtin_bit_cast(f32x4_t, load_piece(part + (first + c) * per + i));
      store_piece(dw + e * per + i, __builtin_bit_cast(u32x4_t, a));
    } else {
      for (int64_t j = i; j < per; ++j) {
        float s = 0.0f;
        for (int64_t c = 0; c < count; ++c) s += part[(first + c) * per + j];
        dw[e * per + j] = s;
      }
    }
  }
  if (db && blockIdx.x == 0) {
    for (int n = threadIdx.x; n < C_out; n += kThreads) {
      float s = 0.0f;
      for (int64_t c = 0; c < count; ++c) s += part_db[(first + c) * C_out + n];
      db[static_cast<int64_t>(e) * C_out + n] = s;
    }
  }
}

// How the weight gradient cuts its groups: chunk = 0 where the groups' own tiles
// fill the card or there is little to sum, else positions per chunk.
struct DwPlan {
  int64_t chunk, jobs;
  size_t bytes;
};
DwPlan dw_plan(int dt, int64_t m, int E, int C_in, int C_out) {
  (void)dt;
  const int64_t tiles = ((C_in + 127ll) / 128) * ((C_out + 127ll) / 128);
  const int64_t want = 1024;                       // workgroups: two waves of two a compute unit
  if (m <= 1024 || E * tiles >= 4 * want) return DwPlan{0, E, 0};
  int64_t chunks = (want + tiles - 1) / tiles;
  int64_t chunk = (m + chunks - 1) / chunks;
  chunk = (chunk + 255) / 256 * 256;
  const int64_t jobs = m / chunk + (E < m ? E : m);
  const size_t per = static_cast<size_t>(C_in) * C_out + C_out;
  return DwPlan{chunk, jobs, static_cast<size_t>(jobs) * per * sizeof(float)};
}

// (a shift of the count: groups never have more tiles than this)
inline int64_t tile_bound(int64_t m, int64_t groups, int64_t BM) {
  return m / BM + (groups < m ? groups : m);
}

template <typename T, typename TO, bool BT, int BM, int BN> int run_tile(GroupedArgs a) {
  const int64_t tiles = tile_bound(a.m, a.E + 1, BM), ncol = (a.cols + BN - 1) / BN;
  // longer strips while they leave four workgroups a compute unit
  int64_t strip = tiles * ncol / 1024;
  strip = strip < 1 ? 1 : strip > ncol ? ncol : strip;
  a.strip = static_cast<int>(strip);
  const int64_t blocks = tiles * ((ncol + strip - 1) / strip);
  if (blocks > 0x7fffffff) return SPCONV_EINVAL;
  const bool whole = a.red % Row<T>::VEC == 0 && (BT || a.cols % Row<T>::VEC == 0);
  if (whole)
    k_grouped<T, TO, BT, BM, BN, true><<<static_cast<uint32_t>(blocks), kThreads, 0, a.st>>>(a);
  else
    k_grouped<T, TO, BT, BM, BN, false><<<static_cast<uint32_t>(blocks), kThreads, 0, a.st>>>(a);
  return launched();
}
template <typename T, typename TO, bool BT> int run_grouped(const GroupedArgs& a) {
  if (a.cols <= 64 || a.m <= 64ll * a.E) return run_tile<T, TO, BT, 64, 64>(a);
  return run_tile<T, TO, BT, 128, 128>(a);
}
template <bool BT> int run_types(int in_dt, int out_dt, const GroupedArgs& a) {
  if (in_dt == SPCONV_BF16)
    return out_dt == SPCONV_BF16 ? run_grouped<bf16_t, bf16_t, BT>(a)
                                 : run_grouped<bf16_t, float, BT>(a);
  return out_dt == SPCONV_BF16 ? run_grouped<float, bf16_t, BT>(a)
                               : run_grouped<float, float, BT>(a);
}

template <typename T, int BC, int BN> void run_dw(const WeightArgs& a, int64_t jobs) {
  const uint32_t blocks = static_cast<uint32_t>(jobs * ((a.C_in + BC - 1) / BC) *
                                                ((a.C_out + BN - 1) / BN));
  if (a.C_in % Row<T>::VEC == 0 && a.C_out % Row<T>::VEC == 0)
    k_grouped_dw<T, BC, BN, true><<<blocks, kThreads, 0, a.st>>>(a);
  else
    k_grouped_dw<T, BC, BN, false><<<blocks, kThreads, 0, a.st>>>(a);
}

bool sizes_ok(int64_t m, int E, int C_in, int C_out) {
  return rows_ok(m) && E >= 1 && E <= 65535 && C_in >= 1 && C_out >= 1 && C_in <= (1 << 23) &&
         C_out <= (1 << 23);
}

}  // namespace
}  // namespace spc

using namespace spc;

extern "C" int spconv_grouped_forward(int in_dt, const void* x, int64_t n_x, const void* w,
                                      const int32_t* offsets, const int32_t* rows,
                                      const float* bias, int relu, int out_dt, void* y, int64_t m,
                                      int E, int C_in, int C_out, void* stream) {
  if (!dtype_ok(in_dt) || !dtype_ok(out_dt) || !sizes_ok(m, E, C_in, C_out) || !rows_ok(n_x) ||
      (relu != 0 && relu != 1) || (!rows && n_x < m))
    return SPCONV_EINVAL;
  const size_t e = elem_bytes(in_dt);
  if (!ptr_ok(x, n_x, e) || !ptr_ok(w, 1, e) || !ptr_ok(offsets, 1, 4) || !aligned_to(rows, 4) ||
      !aligned_to(bias, 4) || !ptr_ok(y, m, elem_bytes(out_dt)))
    return SPCONV_EINVAL;
  if (m == 0) return SPCONV_OK;
  return run_types<false>(in_dt, out_dt,
                          GroupedArgs{x, n_x, w, offsets, rows, bias, nullptr, relu, y, m, E, C_in,
                                      C_out, 1, static_cast<hipStream_t>(stream)});
}

extern "C" int spconv_grouped_backward_data(int dt, const void* dy, const void* w,
                                            const int32_t* offsets, const void* mask, int out_dt,
                                            void* dx, int64_t m, int E, int C_in, int C_out,
                                            void* stream) {
  if (!dtype_ok(dt) || !dtype_ok(out_dt) || !sizes_ok(m, E, C_in, C_out)) return SPCONV_EINVAL;
  const size_t e = elem_bytes(dt), o = elem_bytes(out_dt);
  if (!ptr_ok(dy, m, e) || !ptr_ok(w, 1, e) || !ptr_ok(offsets, 1, 4) || !aligned_to(mask, o) ||
      !ptr_ok(dx, m, o))
    return SPCONV_EINVAL;
  if (m == 0) return SPCONV_OK;
  return run_types<true>(dt, out_dt,
                         GroupedArgs{dy, m, w, offsets, nullptr, nullptr, mask, 0, dx, m, E, C_out,
                                     C_in, 1, static_cast<hipStream_t>(stream)});
}

extern "C" int spconv_grouped_backward_weight_workspace(int dt, int64_t m, int E, int C_in,
                                                        int C_out, size_t* bytes) {
  if (!dtype_ok(dt) || !sizes_ok(m, E, C_in, C_out) || !bytes) return SPCONV_EINVAL;
  *bytes = dw_plan(dt, m, E, C_in, C_out).bytes;
  return SPCONV_OK;
}

extern "C" int spconv_grouped_backward_weight(int dt, const void* x, int64_t n_x, const void* dy,
                                              const int32_t* offsets, const int32_t* rows,
                                              float* dw, float* db, int64_t m, int E, int C_in,
                                              int C_out, void* workspace, size_t workspace_bytes,
                                              void* stream) {
  if (!dtype_ok(dt) || !sizes_ok(m, E, C_in, C_out) || !rows_ok(n_x) || (!rows && n_x < m))
    return SPCONV_EINVAL;
  const size_t e = elem_bytes(dt);
  const DwPlan plan = dw_plan(dt, m, E, C_in, C_out);
  if (!ptr_ok(x, n_x, e) || !ptr_ok(dy, m, e) || !ptr_ok(offsets, 1, 4) || !aligned_to(rows, 4) ||
      !ptr_ok(dw, 1, 4) || !aligned_to(db, 4) ||
      (plan.bytes && (!workspace || !aligned_to(workspace, 16) || workspace_bytes < plan.bytes)))
    return SPCONV_EINVAL;
  const int64_t tiles = ((C_in + 63ll) / 64) * ((C_out + 63ll) / 64);
  if (plan.jobs * tiles > 0x7fffffff) return SPCONV_EINVAL;
  hipStream_t st = static_cast<hipStream_t>(stream);
  WeightArgs a{x, n_x, dy, offsets, rows, dw, db, m, plan.chunk, E, C_in, C_out, st};
  const int64_t per = static_cast<int64_t>(C_in) * C_out;
  if (plan.chunk) {
    a.dw = static_cast<float*>(workspace);
    a.db = db ? a.dw + plan.jobs * per : nullptr;
  }
  const bool small = C_in <= 64 || C_out <= 64;
  if (dt == SPCONV_BF16)
    small ? run_dw<bf16_t, 64, 64>(a, plan.jobs) : run_dw<bf16_t, 128, 128>(a, plan.jobs);
  else
    small ? run_dw<float, 64, 64>(a, plan.jobs) : run_dw<float, 128, 128>(a, plan.jobs);
  if (plan.chunk) {
    const dim3 grid(static_cast<uint32_t>((per + 4 * kThreads - 1) / (4 * kThreads)), E);
    k_grouped_dw_sum<<<grid, kThreads, 0, st>>>(a.dw, a.db, offsets, E, m, plan.chunk, per, C_out,
                                               dw, db);
  }
  return launched();
}
