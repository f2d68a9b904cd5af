// Dense products of feature rows with bias, activation and residual in their epilogue, and
// their gradients, on the matrix cores: rows in bf16, fp32 or 8 bits with a scale a row.
//
// 8-bit rows are multiplied as the bf16 numbers they are (every e4m3 value is one), and the
// row's scale is taken out of the sum: forwards it is a factor of the finished row, in the
// weight gradient, where the sum runs over the rows, it goes to the other operand, scale *
// dy, which enters as the sum of three bf16 numbers.
#include <type_traits>

#include "rows_act.h"
#include "rows_mma.h"
#include "rows_plan.h"

namespace spc {
namespace {

constexpr int kThreads = 256;
constexpr int kSplit = 8;      // slices of the reduction where k_linear has few tiles

struct LinearArgs {
  const void* x;               // [n][red]
  const float* x_scale;        // rows in 8 bits: [n]
  const void* w;
  const float* bias;
  int act;
  const void* side;            // forward: the residual; backward: the activation's input
  const float* side_scale;     // that in 8 bits: [n]
  void *y, *z;                 // [n][cols]
  int64_t n;
  int red, cols;               // reduction, output columns
  hipStream_t st;
  int touch = 0;               // touch_rows
};

// Eight e4m3 values as bf16, exactly.
__device__ __forceinline__ u32x4_t widen(uint32_t lo, uint32_t hi) {
  typedef __bf16 b2 __attribute__((ext_vector_type(2)));
  u32x4_t v;
  v[0] = __builtin_bit_cast(uint32_t, (b2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false));
  v[1] = __builtin_bit_cast(uint32_t, (b2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true));
  v[2] = __builtin_bit_cast(uint32_t, (b2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false));
  v[3] = __builtin_bit_cast(uint32_t, (b2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true));
  return v;
}
// Eight values of an 8-bit row, as load_left.
__device__ __forceinline__ uint2 load8_left(const uint8_t* p, int64_t left) {
  uint2 u = make_uint2(0u, 0u);
  if (left >= 8) {
    __builtin_memcpy(&u, p, 8);
  } else if (left > 0) {
    uint8_t e[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) e[i] = i < left ? p[i] : 0;
    __builtin_memcpy(&u, e, 8);
  }
  return u;
}

// A barrier for what the waves exchange through LDS alone: loads and stores of memory go on
// (__syncthreads waits for them: in the end of every part of a finished tile for its stores).
__device__ __forceinline__ void lds_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xc07f);              // lgkmcnt(0)
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// The finished tile of a workgroup of WR x WC waves, FM x FN blocks each, leaves through LDS
// (BYTES of it) as fp32 rows, a row block of every wave and FNP column blocks at a time:
// everything behind the product is done on fp32 and rounded once, whole rows go to memory, and
// a lane has the same columns for all row blocks (their bias stays in registers).  The
// residual, or the activation's input, is asked for before the barrier that its block's sums
// wait at.
// Forward: z = acc * scale + bias (z is kept if asked for), y = act(z) + residual.
// BT (input gradient): y = acc * act'(side).
// SPLIT: so many groups of WR x WC waves have a slice of the reduction each; their sums are
// added here, in order.
template <typename TO, bool X8, bool BT, int BM, int BN, int WR, int WC, int BYTES, bool PAST,
          int SPLIT = 1>
__device__ __forceinline__ void finish_tile(u32x4_t* lds,
                                            const f32x16 (&acc)[BN / WC / 32][BM / WR / 32],
                                            const LinearArgs& a, int64_t row0, int n0) {
  constexpr int FM = BM / WR / 32, FN = BN / WC / 32, VO = Row<TO>::VEC, NT = 64 * WR * WC * SPLIT;
  constexpr int RW = WR * 32, FNP = RW * BN * 4 * SPLIT <= BYTES ? FN : 1, CW = WC * 32 * FNP;
  constexpr int PR = CW / VO, NPC = RW * PR > NT ? RW * PR / NT : 1, Q = VO / 4;
  constexpr int PART = RW * CW / 4;                // pieces of a slice's part
  static_assert(PART * SPLIT * 16 <= BYTES, "a part of the finished tile fits");
  static_assert(NT % PR == 0 && NPC * NT >= RW * PR, "a lane's pieces lie in the same columns");
  const int slice = threadIdx.x / (64 * WR * WC), wave = (threadIdx.x >> 6) % (WR * WC);
  const int lane = threadIdx.x & 63, h = lane >> 5;
  const int wrow = wave / WC, wcol = wave % WC, piece = threadIdx.x % PR;
  const bool side8 = BT && a.side_scale;
#pragma unroll
  for (int np = 0; np < FN; np += FNP) {
    const int col = n0 + WC * 32 * np + piece * VO, left = a.cols - col;
    float bias[VO];
#pragma unroll
    for (int e = 0; e < VO; ++e) bias[e] = 0.0f;
    if (!BT && a.bias) {
#pragma unroll
      for (int e = 0; e < VO; ++e)
        if (e < left) bias[e] = a.bias[col + e];
    }
#pragma unroll
    for (int m = 0; m < FM; ++m) {
      u32x4_t g[NPC];
      float xs[NPC];
      int64_t at[NPC];
      bool live[NPC];
#pragma unroll
      for (int i = 0; i < NPC; ++i) {
        const int lr = (threadIdx.x + NT * i) / PR;
        const int64_t r = row0 + lr / 32 * (BM / WR) + 32 * m + lr % 32;
        live[i] = r < a.n && left > 0 && (NPC * NT == RW * PR || lr < RW);
        at[i] = r * a.cols + col;
        xs[i] = X8 && live[i] ? a.x_scale[r] : 1.0f;
        if (a.side && live[i]) {
          if (side8) {
            const uint2 u = load8_left(static_cast<const uint8_t*>(a.side) + at[i],
                                       left < VO ? left : VO);
            g[i][0] = u.x, g[i][1] = u.y;
            xs[i] = a.side_scale[r];
          } else {
            g[i] = load_left<TO, false>(static_cast<const TO*>(a.side) + at[i], left);
          }
        }
      }
      lds_barrier();
#pragma unroll
      for (int f = 0; f < FNP; ++f)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          // 4 adjacent columns of one row in every four registers of a lane
          const int c = col_of<WC>(wcol, f) + 8 * q + 4 * h;
          u32x4_t v;
#pragma unroll
          for (int i = 0; i < 4; ++i) v[i] = __float_as_uint(acc[np + f][m][4 * q + i]);
          lds[slice * PART + out_at<float, CW>(wrow * 32 + (lane & 31), c / 4)] = v;
        }
      lds_barrier();
#pragma unroll
      for (int i = 0; i < NPC; ++i) {
        if (!live[i]) continue;
        const int lr = (threadIdx.x + NT * i) / PR;
        float v[VO];
#pragma unroll
        for (int q = 0; q < Q; ++q) {
          const int at = out_at<float, CW>(lr, piece * Q + q);
          const u32x4_t u = lds[at];
#pragma unroll
          for (int e = 0; e < 4; ++e) v[4 * q + e] = __uint_as_float(u[e]);
#pragma unroll
          for (int p = 1; p < SPLIT; ++p) {
            const u32x4_t more = lds[p * PART + at];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[4 * q + e] += __uint_as_float(more[e]);
          }
        }
        if constexpr (BT) {
          if (a.side) {
            float s[VO];
            if (side8) {
#pragma unroll
              for (int q = 0; q < Q; ++q) unpack_e4m3(g[i][q], s + 4 * q);
#pragma unroll
              for (int e = 0; e < VO; ++e) s[e] *= xs[i];
            } else {
              unpack(g[i], s);
            }
            by_act(a.act, [&](auto k) {
#pragma unroll
              for (int e = 0; e < VO; ++e) v[e] *= slope<decltype(k)::value, sizeof(TO) == 4>(s[e]);
            });
          }
        } else {
#pragma unroll
          for (int e = 0; e < VO; ++e) v[e] = X8 ? v[e] * xs[i] + bias[e] : v[e] + bias[e];
          if (a.z) store_left<TO, PAST>(static_cast<TO*>(a.z) + at[i], pack(v), left);
          by_act(a.act, [&](auto k) {
#pragma unroll
            for (int e = 0; e < VO; ++e) v[e] = activate<decltype(k)::value, sizeof(TO) == 4>(v[e]);
          });
          if (a.side) {
            float s[VO];
            unpack(g[i], s);
#pragma unroll
            for (int e = 0; e < VO; ++e) v[e] += s[e];
          }
        }
        store_left<TO, PAST>(static_cast<TO*>(a.y) + at[i], pack(v), left);
      }
    }
  }
}

// A workgroup's tile: rows from row0, columns from n0 (the column tiles of one row tile side by
// side on one die, whose L2 then has their rows).
struct TileAt {
  int64_t row0;
  int n0;
};
template <int BM, int BN> __device__ __forceinline__ TileAt tile_at(int cols) {
  const int ncol = (cols + BN - 1) / BN;
  const int64_t id = die_order(blockIdx.x, gridDim.x);
  return TileAt{id / ncol * BM, static_cast<int>(id % ncol) * BN};
}

// Rows of BK e4m3 values in LDS, as RTile; a fragment is 8 bytes, widened when it is read.
template <int R, int BK> struct RTile8 {
  static constexpr int PR = BK / 16, PIECES = R * PR;      // (a piece is a step of the reduction)
  __device__ static int at(int row, int piece) {
    return row * PR + (piece ^ (PR == 4 ? (row >> 2) & 3 : (row >> 3) & 1));
  }
  struct Reader {
    int place[PR];
    __device__ Reader(int r0, int lane) {
#pragma unroll
      for (int s = 0; s < PR; ++s)
        place[s] = lane_place(at(r0 + (lane & 31), s) * 16 + 8 * (lane >> 5));
    }
    __device__ bf16x8 operator()(const u32x4_t* t, int b, int s) const {
      const uint2 u = lds_at<uint2>(t, place[s] + b * 32 * BK);
      return __builtin_bit_cast(bf16x8, widen(u.x, u.y));
    }
  };
};

// Workgroups of a die that run together.
template <int BM> constexpr int kResident = BM == 256 ? 64 : BM == 128 ? 96 : 160;
// The first 4 bytes of every line of this workgroup's share of the rows that will be read `ahead`
// tiles on by this die, into its L2 (and, unread, into LDS at `room`, 256 bytes a wave): the
// column tiles of one row tile run side by side and would all wait for its rows, three stages of
// them at a time.  To be waited for before the workgroup ends.
template <int BM, int BN, int NT>
__device__ __forceinline__ void touch_rows(const void* x, int64_t row_bytes, int64_t n, int cols,
                                           int ahead, u32x4_t* room) {
  const int64_t total = gridDim.x, local = blockIdx.x / 8, die = blockIdx.x % 8;
  if (local + ahead >= total / 8 + (die < total % 8)) return;
  const int ncol = (cols + BN - 1) / BN;
  const int64_t id = die_order(blockIdx.x, total) + ahead, row0 = id / ncol * BM;
  const int64_t bytes = (n - row0 < BM ? n - row0 : BM) * row_bytes;
  // (whole lines from the tile's first byte on, and so whole words inside it)
  const int64_t share = (bytes + 128ll * ncol - 1) / (128ll * ncol) * 128, first = id % ncol * share;
  const int64_t end = first + share < bytes ? first + share : bytes;
  typedef __attribute__((address_space(3))) void lds_void;
  typedef __attribute__((address_space(1))) const void global_void;
  const char* const p = static_cast<const char*>(x) + row0 * row_bytes;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  for (int64_t at = first + threadIdx.x * 128; at < end; at += NT * 128)
    __builtin_amdgcn_global_load_lds((global_void*)(p + at), (lds_void*)(room + 16 * wave), 4, 0, 0);
}

// Rows x weights of whole aligned 16-byte pieces: BT false: w is [red][cols] (the forward), BT
// true: w is [cols][red] (the input gradient).  A workgroup of WR x WC waves takes a tile of BM
// rows by BN columns, in stages of BK of the reduction through a ring of LDS buffers: all but
// one stage are on their way while that one is multiplied, one barrier a stage.
// SPLIT: so many groups of WR x WC waves, each with a slice of the reduction and buffers of its own:
// where there are few tiles the stages of one follow each other in time, and nothing else
// runs on the card (64 x 2048 -> 512 bf16: 14.1 us, in eight slices 6.5).
// Of the cycles a compute unit has work, the matrix cores are busy in 45 % and the LDS in 25 (16,384 x
// 2048 -> 2048 bf16: 145 us, 950 TFLOP/s, a large library product 1,147), or in 19 and 17 (348,208 x
// 256 -> 1024 with the activation's input, 411 us with its rows in the last-level cache and 461
// without, 3.9 and 3.5 TB/s: eight stages a tile, whose first ones wait for memory; what
// k_linear_short does not take, 8-bit and fp32 rows or sums, runs so).  (256 x
// 128 by four waves instead of eight, 128 x 256, 256 x 256: 5 to 10 % slower; a ring of four: an
// LDS' worth of workgroups fewer, 20 %; the residual asked for a tile ahead: registers for
// one workgroup a compute unit instead of two, 25 %.)
template <typename T, typename TO, bool X8, bool BT, int BM, int BN, int WR, int WC, bool PAST,
          int SPLIT>
__global__ __launch_bounds__(64 * WR * WC * SPLIT, 2) void k_linear(LinearArgs a) {
  // (rows in 8 bits: 64 of them are too few pieces for the lanes in stages of 32)
  constexpr int KB = X8 && BM == 64 ? 128 : 64, BK = kBK<T, KB>, NT = 64 * WR * WC;
  constexpr int kRing = 3;
  typedef std::conditional_t<X8, RTile8<BM, BK>, RTile<T, BM, KB>> TA;
  typedef RTile<T, BN, KB> TBr;
  typedef KTile<T, BN, KB> TBk;
  constexpr int VEC = Row<T>::VEC, VX = X8 ? 16 : VEC;     // elements of a piece
  constexpr int FM = BM / WR / 32, FN = BN / WC / 32;
  constexpr int PA = TA::PIECES / NT, PB = TBk::PIECES / NT;
  constexpr int NP = TA::PIECES + TBk::PIECES;
  static_assert(PA * NT == TA::PIECES && PB * NT == TBk::PIECES, "whole pieces a lane");
  // (the first one also takes the finished tile; separate arrays, so that the compiler
  // knows which loads a read waits for)
  constexpr int kOut = WR * 32 * WC * 32 / 4, NP0 = kOut > NP ? kOut : NP;
  __shared__ u32x4_t s_buf0[NP0 * SPLIT], s_buf1[NP * SPLIT], s_buf2[NP * SPLIT];
  typedef std::conditional_t<X8, uint8_t, T> TX;
  static_assert(NP >= 16 * (NT / 64), "room for what touch_rows brings");
  const TX* const x = static_cast<const TX*>(a.x);
  const T* const w = static_cast<const T*>(a.w);
  const TileAt t = tile_at<BM, BN>(a.cols);
  // (of a slice of the reduction; its buffers are the slice's part of each)
  const int slice = SPLIT > 1 ? threadIdx.x / NT : 0, tid = threadIdx.x - slice * NT;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = threadIdx.x & 63;
  const int ours = __builtin_amdgcn_readfirstlane(slice * NP);
  const int nk = (a.red + BK * SPLIT - 1) / (BK * SPLIT);    // stages of a slice
  const int k0 = slice * nk * BK, kend = k0 + nk * BK < a.red ? k0 + nk * BK : a.red;

  // What this lane stages of the rows: rows ra0 + NT / PR * i, of each the piece that
  // belongs at its place in LDS.  A row that is not there is read as zeros, at one place all
  // along (step 0).
  constexpr int PRA = TA::PR, PRB = TBr::PR;
  static_assert(NT / PRA % 16 == 0 && NT / PRB % 16 == 0, "a lane's pieces have one place in their rows");
  const int ra0 = tid / PRA, ka = (TA::at(ra0, tid % PRA) - ra0 * PRA) * VX;
  const TX* const zero = reinterpret_cast<const TX*>(&g_zeros);
  const TX* pa[PA];
  int step[PA];
#pragma unroll
  for (int i = 0; i < PA; ++i) {
    const int64_t r = t.row0 + ra0 + NT / PRA * i;
    step[i] = r < a.n ? BK : 0;
    pa[i] = r < a.n ? x + r * a.red + k0 + ka : zero;
  }
  // And of the weights, from the stage's own place; columns past the last one are read as
  // others (nothing of them is stored).
  const int kb = BT ? tid / PRB : tid / TBk::PR;
  const int kr = BT ? (TBr::at(kb, tid % PRB) - kb * PRB) * VEC : 0;
  uint32_t pb[PB];
#pragma unroll
  for (int i = 0; i < PB; ++i) {
    if constexpr (BT) {
      const int n = kb + NT / PRB * i;
      pb[i] = static_cast<uint32_t>(t.n0 + n < a.cols ? n : 0) * a.red + kr;
    } else {
      const int n = (TBk::at(kb, tid % TBk::PR) - kb * TBk::PR) * VEC;
      pb[i] = static_cast<uint32_t>(kb + NT / TBk::PR * i) * a.cols + (t.n0 + n < a.cols ? n : 0);
    }
  }
  // Stages past the last one are asked for too, as zeros, so that the number of loads
  // behind a stage's own is known.
  int rk = k0;                                     // the next stage to request
  auto request = [&](u32x4_t* buf) {
    buf += ours;
    const int left = kend - rk;                    // of the slice
    const T* const ws = BT ? w + static_cast<int64_t>(t.n0) * a.red + rk
                           : w + static_cast<int64_t>(rk) * a.cols + t.n0;
    if (left >= BK) {
#pragma unroll
      for (int i = 0; i < PA; ++i) {
        load_to_lds(pa[i], buf + NT * i + 64 * wave);
        pa[i] += step[i];
      }
#pragma unroll
      for (int i = 0; i < PB; ++i)
        load_to_lds(ws + pb[i], buf + TA::PIECES + NT * i + 64 * wave);
    } else {
#pragma unroll
      for (int i = 0; i < PA; ++i)
        load_to_lds(ka < left ? pa[i] : zero, buf + NT * i + 64 * wave);
#pragma unroll
      for (int i = 0; i < PB; ++i)
        load_to_lds((BT ? kr : kb + NT / TBk::PR * i) < left
                        ? static_cast<const void*>(ws + pb[i]) : &g_zeros,
                    buf + TA::PIECES + NT * i + 64 * wave);
    }
    rk += BK;
  };

  const typename TA::Reader rows_of(wave / WC * (BM / WR), lane);
  const std::conditional_t<BT, typename TBr::Reader, typename TBk::template Reader<32 * WC, FN>>
      weights_of(32 * (wave % WC), lane);
  f32x16 acc[FN][FM];
#pragma unroll
  for (int n = 0; n < FN; ++n)
#pragma unroll
    for (int m = 0; m < FM; ++m)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[n][m][i] = 0.0f;
  auto stage = [&](const u32x4_t* buf, u32x4_t* before) {
    stage_barrier<(PA + PB) * (kRing - 2)>();
    request(before);
    multiply_stage<T, KB, FM, FN>(
        acc, [&](int m, int q) { return rows_of(buf + ours, m, q); },
        [&](int n, int q) { return weights_of(buf + ours + TA::PIECES, BT ? WC * n : n, q); });
  };
  request(s_buf0);
  request(s_buf1);
  for (int s = 0; s < nk; s += kRing) {
    stage(s_buf0, s_buf2);
    if (s + 1 < nk) stage(s_buf1, s_buf0);
    if (s + 2 < nk) stage(s_buf2, s_buf1);
  }
  stage_barrier<0>();                              // (no load is on its way to s_buf0)
  if (a.touch && SPLIT == 1)
    touch_rows<BM, BN, NT>(a.x, static_cast<int64_t>(a.red) * sizeof(TX), a.n, a.cols,
                           kResident<BM>, s_buf1);
  finish_tile<TO, X8, BT, BM, BN, WR, WC, NP0 * SPLIT * 16, PAST, SPLIT>(s_buf0, acc, a, t.row0,
                                                                        t.n0);
  if (a.touch && SPLIT == 1) stage_barrier<0>();
}

// bf16 rows, a reduction of at most 32 NK, nothing read behind it but a residual: a workgroup keeps the weights
// of its 256 columns in registers (four waves of 64 columns, twice, for 32 rows each) while rows
// stream past it, 64 at a time through a ring of three LDS buffers.  One barrier a tile is all, and
// its stores are on their way while the next ones are computed: sums leave rounded, wave by wave,
// through LDS of the wave's own, in whole lines of 64 columns.  (Waves of 32 columns, whose stores
// are half lines, take twice the time at 262,144 x 128 -> 272 with the activation's input: 193
// us, and 89.)  A wave's loads and stores are counted together, in their order: behind the loads of
// the tile that is needed next lie the next tile's and, where all of a wave's columns are there,
// the stores and the next residual's loads of the tile before.  (An activation's input read in the
// same way, for the input gradient, takes more registers than there are: 348,208 x 256 -> 1024 616
// us, k_linear 539.)  Bound by memory: 348,208 x 256 -> 1024 220 us (4.1 TB/s), with
// the activation's input 345 (4.6 TB/s), a residual 352 (4.6 TB/s), 1024 <- 256 backwards 212
// (4.2 TB/s); k_linear 334, 411, 488 and 295.  Matrix cores and LDS are busy in 23 % of the cycles
// each, the vector ALU (activating) in 40.
template <bool BT, int NK, bool PAST, bool RES>
__global__ __launch_bounds__(512, NK == 2 && !RES ? 4 : 2) void k_linear_short(LinearArgs a, int strips) {
  typedef bf16_t T;
  typedef Mma<T> M;
  typedef RTile<T, 64, 64> TA;                     // 64 rows, 32 of the reduction
  constexpr int BM = 64, FN = 2, VEC = 8, SUB = TA::PIECES, NP = SUB * NK, PA = NP / 512;
  static_assert(PA * 512 == NP, "whole pieces a lane");
  __shared__ u32x4_t s_buf0[NP], s_buf1[NP], s_buf2[NP], s_out[8][32 * 64 / 8];
  __shared__ __attribute__((aligned(16))) float s_bias[BT ? 4 : 256];
  const T *const x = static_cast<const T*>(a.x), *const w = static_cast<const T*>(a.w);
  const int groups = (a.cols + 255) / 256;
  const int64_t id = die_order(blockIdx.x, gridDim.x);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, h = lane >> 5;
  const int c0 = static_cast<int>(id % groups) * 256 + wave % 4 * 64, r0 = wave / 4 * 32;
  const int64_t tiles = (a.n + BM - 1) / BM;
  const T* const zero = reinterpret_cast<const T*>(&g_zeros);

  // This lane's pieces of a tile: row ra of sub-tiles j0, j0 + 2, ..., the piece whose place in LDS
  // is the lane's.
  constexpr int PRA = TA::PR;
  const int ra = threadIdx.x % SUB / PRA, ka = (TA::at(ra, threadIdx.x % PRA) - ra * PRA) * VEC;
  const int j0 = threadIdx.x / SUB;
  auto request = [&](int64_t t, u32x4_t* buf) {
    const int64_t r = t * BM + ra;
    const T* const p = x + r * a.red + ka;
#pragma unroll
    for (int i = 0; i < PA; ++i) {
      const int k = (j0 + 2 * i) * 32;
      load_to_lds(t < tiles && r < a.n && k + ka < a.red ? p + k : zero, buf + 512 * i + 64 * wave);
    }
  };
  int64_t t = id / groups;
  request(t, s_buf0);
  request(t + strips, s_buf1);

  // Its weights, 64 of the reduction at a time through s_out.
  typename M::Frag fw[FN][2 * NK];
  {
    typedef RTile<T, 256, 128> TR;                 // BT: rows of weights are columns of y
    typedef KTile<T, 256, 128> TK;
    static_assert(TR::PIECES == 2048 && TK::PIECES == 2048 && NK % 2 == 0, "s_out");
    const int base = c0 - wave % 4 * 64;
    u32x4_t raw[2 * NK];
#pragma unroll
    for (int i = 0; i < 2 * NK; ++i) {
      const int piece = threadIdx.x + 512 * (i % 4);
      if constexpr (BT) {
        const int n = base + piece / 8, k = i / 4 * 64 + piece % 8 * 8;
        raw[i] = load_left<T, true>(w + static_cast<int64_t>(n) * a.red + k, n < a.cols ? a.red - k : 0);
      } else {
        const int k = i / 4 * 64 + piece / 32, n = base + piece % 32 * 8;
        raw[i] = load_left<T, true>(w + static_cast<int64_t>(k) * a.cols + n, k < a.red ? a.cols - n : 0);
      }
    }
    if (!BT && threadIdx.x < 256) {
      const int n = base + threadIdx.x;
      s_bias[threadIdx.x] = a.bias && n < a.cols ? a.bias[n] : 0.0f;
    }
    const auto weights_of = [&] {
      if constexpr (BT) return typename TR::Reader(wave % 4 * 64, lane);
      else return typename TK::template Reader<32, FN>(wave % 4 * 64, lane);
    }();
#pragma unroll
    for (int part = 0; part < NK / 2; ++part) {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int piece = threadIdx.x + 512 * i;
        s_out[0][BT ? TR::at(piece / 8, piece % 8) : TK::at(piece / 32, piece % 32)] = raw[4 * part + i];
      }
      __syncthreads();
#pragma unroll
      for (int s = 0; s < 4; ++s)
#pragma unroll
        for (int b = 0; b < FN; ++b) fw[b][4 * part + s] = weights_of(s_out[0], b, s);
    }
  }
  // It stores rows lane / 8 + 8 j of a wave's 32, eight columns.  In LDS pieces are permuted by
  // pairs of rows, their halves exchanged from row 16 on: writes of half a piece by 32 rows and
  // reads of whole ones meet every bank once.
  const int col = c0 + lane % 8 * 8, left = a.cols - col;
  constexpr int kStores = 4;                       // of a tile, twice as many with z
  constexpr int kSide = RES ? 4 : 0;               // loads of the residual
  const bool whole = c0 + 64 <= a.cols;            // (one for the wave)
  u32x4_t* const out = s_out[wave];
  const int put = (lane & 31) * 128 + (h ^ (lane >> 4 & 1)) * 8, turn = lane >> 1 & 7;
  const typename TA::Reader rows_of(r0, lane);

  // The next tile's residual, in the places that are stored.
  u32x4_t res[4];
  auto res_of = [&](int64_t t) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int64_t r = t * BM + r0 + lane / 8 + 8 * j;
      const T* const p = static_cast<const T*>(a.side) + r * a.cols + col;
      res[j] = load_left<T, true>(p, r < a.n ? left : 0);
    }
  };
  if constexpr (RES) res_of(t);

  auto tile = [&](const u32x4_t* buf, u32x4_t* before) {
    if (!whole) stage_barrier<PA>();
    else if (a.z) stage_barrier<PA + 2 * kStores + kSide>();
    else stage_barrier<PA + kStores + kSide>();
    request(t + 2 * strips, before);
    asm volatile("" ::: "memory");                 // (the tile's stores come behind these loads)
    f32x16 acc[FN];
#pragma unroll
    for (int b = 0; b < FN; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[b][i] = 0.0f;
#pragma unroll
    for (int q = 0; q < 2 * NK; ++q) {
      const typename M::Frag fa = rows_of(buf + q / 2 * SUB, 0, q % 2);
#pragma unroll
      for (int b = 0; b < FN; ++b) acc[b] = M::mma(fw[b][q], fa, acc[b]);
    }
    auto leave = [&](void* y) {
#pragma unroll
      for (int b = 0; b < FN; ++b)
#pragma unroll
        for (int q = 0; q < 4; q += 2) {
          float v[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) v[i] = acc[b][4 * q + i];
          const u32x4_t u = pack(v);
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const uint2 half = {u[2 * i], u[2 * i + 1]};
            *reinterpret_cast<uint2*>(reinterpret_cast<char*>(out) + put + ((4 * b + q + i) ^ turn) * 16) = half;
          }
        }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int lr = lane / 8 + 8 * j;
        const int64_t r = t * BM + r0 + lr;
        if (r >= a.n || left <= 0) continue;
        u32x4_t u = out[lr * 8 + (lane % 8 ^ (lr >> 1 & 7))];
        if (j >= 2) u = u32x4_t{u[2], u[3], u[0], u[1]};
        store_left<T, PAST>(static_cast<T*>(y) + r * a.cols + col, u, left);
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    };
    if constexpr (!BT) {
      // (a lane's sums are of row lane % 32, columns 32 b + 8 q + 4 h + i)
#pragma unroll
      for (int b = 0; b < FN; ++b)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const float4 v = *reinterpret_cast<const float4*>(s_bias + wave % 4 * 64 + 32 * b + 8 * q + 4 * h);
          acc[b][4 * q] += v.x, acc[b][4 * q + 1] += v.y, acc[b][4 * q + 2] += v.z, acc[b][4 * q + 3] += v.w;
        }
      if (a.z) leave(a.z);
      by_act(a.act, [&](auto k) {
#pragma unroll
        for (int b = 0; b < FN; ++b)
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[b][i] = activate<decltype(k)::value, false>(acc[b][i]);
      });
    }
    if constexpr (RES) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int lr = lane / 8 + 8 * j;
        u32x4_t u = res[j];
        if (j >= 2) u = u32x4_t{u[2], u[3], u[0], u[1]};
        out[lr * 8 + (lane % 8 ^ (lr >> 1 & 7))] = u;
      }
      res_of(t + strips);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int b = 0; b < FN; ++b)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const uint2 u = *reinterpret_cast<const uint2*>(reinterpret_cast<const char*>(out) + put +
                                                          ((4 * b + q) ^ turn) * 16);
          acc[b][4 * q] += __uint_as_float(u.x << 16);
          acc[b][4 * q + 1] += __uint_as_float(u.x & 0xffff0000u);
          acc[b][4 * q + 2] += __uint_as_float(u.y << 16);
          acc[b][4 * q + 3] += __uint_as_float(u.y & 0xffff0000u);
        }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
    leave(a.y);
    t += strips;
  };
  // (Before the first tile nothing was stored.)
  stage_barrier<0>();
  while (t < tiles) {
    tile(s_buf0, s_buf2);
    if (t < tiles) tile(s_buf1, s_buf0);
    if (t < tiles) tile(s_buf2, s_buf1);
  }
  stage_barrier<0>();                              // (no load to LDS outlives the workgroup)
}

// Rows x weights for any alignment and width: BT false: w is [red][cols] (the forward), BT true:
// w is [cols][red] (the input gradient).  Through registers, 128 x 128 or 64 x 64 by four
// waves in 2 x 2, stages of 128 bytes of the reduction.  X8: rows in 8 bits, widened on their
// way to LDS.  Bound by the time from a stage's loads to its products, one stage at a time (60,000 x
// 145 -> 301 bf16: 33 us, 158 TFLOP/s).
template <typename T, typename TO, bool X8, bool BT, int BM, int BN>
__global__ __launch_bounds__(kThreads, 2) void k_linear_any(LinearArgs a) {
  constexpr int KB = 128;
  typedef RTile<T, BM, KB> TA;
  typedef RTile<T, BN, KB> TBr;
  typedef KTile<T, BN, KB> TBk;
  constexpr int VEC = Row<T>::VEC, BK = kBK<T, KB>;
  constexpr int FM = BM / 64, FN = BN / 64;
  constexpr int PA = TA::PIECES / kThreads, PB = TBk::PIECES / kThreads;
  constexpr int NP = TA::PIECES + TBk::PIECES;
  __shared__ u32x4_t s_buf[NP];
  const TileAt t = tile_at<BM, BN>(a.cols);
  const int64_t row0 = t.row0;
  const int n0 = t.n0;
  const T* const w = static_cast<const T*>(a.w);
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int ra0 = threadIdx.x >> 3, ka = (threadIdx.x & 7) * VEC;
  u32x4_t ra[PA], rb[PB];
  auto request = [&](int k0) {
#pragma unroll
    for (int i = 0; i < PA; ++i) {
      const int64_t r = row0 + ra0 + 32 * i;
      const int left = r < a.n ? a.red - k0 - ka : 0;
      if constexpr (X8) {
        const uint2 u = load8_left(static_cast<const uint8_t*>(a.x) + r * a.red + k0 + ka, left);
        ra[i] = widen(u.x, u.y);
      } else {
        ra[i] = load_left<T, false>(static_cast<const T*>(a.x) + r * a.red + k0 + ka, left);
      }
    }
#pragma unroll
    for (int i = 0; i < PB; ++i) {
      if constexpr (BT) {
        const int n = n0 + ra0 + 32 * i;
        rb[i] = load_left<T, false>(w + static_cast<int64_t>(n) * a.red + k0 + ka,
                                    n < a.cols ? a.red - k0 - ka : 0);
      } else {
        const int p = threadIdx.x + kThreads * i;
        const int k = k0 + p / TBk::PR, n = n0 + p % TBk::PR * VEC;
        rb[i] = load_left<T, false>(w + static_cast<int64_t>(k) * a.cols + n,
                                    k < a.red ? a.cols - n : 0);
      }
    }
  };
  const typename TA::Reader rows_of((wave >> 1) * (BM / 2), lane);
  const std::conditional_t<BT, typename TBr::Reader, typename TBk::template Reader<64, FN>>
      weights_of(32 * (wave & 1), lane);
  f32x16 acc[FN][FM];
#pragma unroll
  for (int n = 0; n < FN; ++n)
#pragma unroll
    for (int m = 0; m < FM; ++m)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[n][m][i] = 0.0f;
  request(0);
  for (int k0 = 0; k0 < a.red; k0 += BK) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < PA; ++i) s_buf[TA::at(ra0 + 32 * i, threadIdx.x & 7)] = ra[i];
#pragma unroll
    for (int i = 0; i < PB; ++i) {
      const int p = threadIdx.x + kThreads * i;
      s_buf[TA::PIECES + (BT ? TBr::at(ra0 + 32 * i, threadIdx.x & 7)
                             : TBk::at(p / TBk::PR, p % TBk::PR))] = rb[i];
    }
    __syncthreads();
    if (k0 + BK < a.red) request(k0 + BK);
    multiply_stage<T, KB, FM, FN>(
        acc, [&](int m, int q) { return rows_of(s_buf, m, q); },
        [&](int n, int q) { return weights_of(s_buf + TA::PIECES, BT ? 2 * n : n, q); });
  }
  finish_tile<TO, X8, BT, BM, BN, 2, 2, NP * 16, false>(s_buf, acc, a, row0, n0);
}

// Few fp32 rows (one at a time): the weights' bytes, once, and the time to the last of them are all
// there is.  A workgroup of 16 waves takes up to 4 rows and 64 bytes of columns, 4 lanes
// side by side; its 256 slices of the reduction run down the weights' rows on the vector ALU,
// 8 loads of a slice in flight, and are added over the lanes, then the waves, in order.
// (1 row 2048 -> 512: 5.6 us, in sliced tiles on the matrix cores 14.5: they take 64 cycles
// for 2 of the reduction however few rows there are.)
constexpr int kFewThreads = 1024, kFewRows = 4;
template <typename TO>
__global__ __launch_bounds__(kFewThreads) void k_linear_few(LinearArgs a) {
  typedef float T;
  constexpr int VEC = Row<T>::VEC, R = kFewRows, CL = 4, NC = CL * VEC, KS = kFewThreads / CL;
  constexpr int KC = 2048, UN = 8;                 // of the reduction in LDS; loads in flight
  static_assert(KS * UN == KC, "a slice's loads reach to the end of what is in LDS");
  constexpr int NW = kFewThreads / 64;
  __shared__ float s_x[R][KC];
  __shared__ float s_sum[NW][R][NC];
  const T* const w = static_cast<const T*>(a.w);
  const TileAt t = tile_at<R, NC>(a.cols);
  const int slice = threadIdx.x / CL, c = t.n0 + threadIdx.x % CL * VEC;
  float acc[R][VEC];
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int i = 0; i < VEC; ++i) acc[r][i] = 0.0f;
  const int sr = threadIdx.x / (kFewThreads / R);  // the row a lane stages
  const int64_t src = t.row0 + sr;
  for (int k0 = 0; k0 < a.red; k0 += KC) {
    const int kc = a.red - k0 < KC ? a.red - k0 : KC;
    u32x4_t u[UN];
    // (on their way while the rows are staged)
#pragma unroll
    for (int i = 0; i < UN; ++i) {
      const int k = slice + KS * i;
      u[i] = load_piece(k < kc && c < a.cols ? w + static_cast<int64_t>(k0 + k) * a.cols + c
                                             : reinterpret_cast<const T*>(&g_zeros));
    }
    __syncthreads();
    for (int k = threadIdx.x % (kFewThreads / R); k < kc; k += kFewThreads / R) {
      float v = 0.0f;
      if (src < a.n) {
        v = static_cast<const T*>(a.x)[src * a.red + k0 + k];
      }
      s_x[sr][k] = v;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < UN; ++i) {
      const int k = slice + KS * i;
      if (k >= kc) break;
      float v[VEC];
      unpack(u[i], v);
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int e = 0; e < VEC; ++e) acc[r][e] = fmaf(s_x[r][k], v[e], acc[r][e]);
    }
  }
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      float v = acc[r][e];
      v += row_rotate<8>(v);
      v += row_rotate<4>(v);
      const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false,
                                                      false);
      v = __uint_as_float(p[0]) + __uint_as_float(p[1]);
      const auto q = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false,
                                                      false);
      v = __uint_as_float(q[0]) + __uint_as_float(q[1]);
      if (lane < CL) s_sum[wave][r][lane * VEC + e] = v;
    }
  __syncthreads();
  if (threadIdx.x >= R * NC) return;
  const int r = threadIdx.x / NC, col = t.n0 + threadIdx.x % NC;
  if (t.row0 + r >= a.n || col >= a.cols) return;
  const int64_t at = (t.row0 + r) * a.cols + col;
  float z = 0.0f;
#pragma unroll
  for (int q = 0; q < NW; ++q) z += s_sum[q][r][threadIdx.x % NC];
  if (a.bias) z += a.bias[col];
  if (a.z) static_cast<TO*>(a.z)[at] = Row<TO>::put(z);
  by_act(a.act, [&](auto k) { z = activate<decltype(k)::value, sizeof(TO) == 4>(z); });
  if (a.side) z += Row<TO>::get(static_cast<const TO*>(a.side)[at]);
  static_cast<TO*>(a.y)[at] = Row<TO>::put(z);
}

// The same for the input gradient, where a row of weights is the reduction: a wave takes two of
// them, its lanes side by side along them, and adds the lanes up at the end.  (2048 -> 512: 3.3 us;
// sliced tiles 5.7.)
template <typename TO>
__global__ __launch_bounds__(kThreads) void k_linear_few_back(LinearArgs a) {
  typedef float T;
  constexpr int VEC = Row<T>::VEC, R = kFewRows, NC = 2, KC = 2048;
  __shared__ __attribute__((aligned(16))) float s_x[R][KC];
  const T *const x = static_cast<const T*>(a.x), *const w = static_cast<const T*>(a.w);
  const TileAt t = tile_at<R, NC * kThreads / 64>(a.cols);
  const int lane = threadIdx.x & 63, c0 = t.n0 + static_cast<int>(threadIdx.x >> 6) * NC;
  float acc[NC][R];
#pragma unroll
  for (int n = 0; n < NC; ++n)
#pragma unroll
    for (int r = 0; r < R; ++r) acc[n][r] = 0.0f;
  for (int k0 = 0; k0 < a.red; k0 += KC) {
    const int kc = a.red - k0 < KC ? a.red - k0 : KC;
    __syncthreads();
    for (int k = threadIdx.x; k < kc; k += kThreads)
#pragma unroll
      for (int r = 0; r < R; ++r)
        s_x[r][k] = t.row0 + r < a.n ? Row<T>::get(x[(t.row0 + r) * a.red + k0 + k]) : 0.0f;
    __syncthreads();
#pragma unroll 4
    for (int k = lane * VEC; k < kc; k += 64 * VEC) {
      float v[NC][VEC];
#pragma unroll
      for (int n = 0; n < NC; ++n)
        unpack(load_piece(c0 + n < a.cols ? w + static_cast<int64_t>(c0 + n) * a.red + k0 + k
                                          : reinterpret_cast<const T*>(&g_zeros)), v[n]);
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int e = 0; e < VEC; e += 4) {
          const float4 d = *reinterpret_cast<const float4*>(&s_x[r][k + e]);
#pragma unroll
          for (int n = 0; n < NC; ++n) {
            acc[n][r] = fmaf(d.x, v[n][e], acc[n][r]);
            acc[n][r] = fmaf(d.y, v[n][e + 1], acc[n][r]);
            acc[n][r] = fmaf(d.z, v[n][e + 2], acc[n][r]);
            acc[n][r] = fmaf(d.w, v[n][e + 3], acc[n][r]);
          }
        }
    }
  }
  float mine = 0.0f;                               // lane r NC + n: row r, column n
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int n = 0; n < NC; ++n) {
      const float v = group_sum<64>(acc[n][r]);
      mine = lane == r * NC + n ? v : mine;
    }
  const int64_t row = t.row0 + lane / NC;
  const int col = c0 + lane % NC;
  if (lane >= R * NC || row >= a.n || col >= a.cols) return;
  const int64_t at = row * a.cols + col;
  if (a.side) {
    float z;
    if (a.side_scale)
      z = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<const uint8_t*>(a.side)[at], false)[0] *
          a.side_scale[row];
    else
      z = Row<TO>::get(static_cast<const TO*>(a.side)[at]);
    by_act(a.act, [&](auto k) { mine *= slope<decltype(k)::value, sizeof(TO) == 4>(z); });
  }
  static_cast<TO*>(a.y)[at] = Row<TO>::put(mine);
}

// Weight gradient of a BC x BN tile over a chunk of the rows: dw[c][n] = sum_j x[j][c] dy[j][n],
// the rows staged as the reduction.  Chunk `job` leaves its sums as part[job]; the workgroups of
// the first rows of dw also sum dy.  No atomics: the chunks are added in their order.
struct LinearWeight {
  const void* x;
  const float* x_scale;
  const void* dy;
  float *dw, *db;              // where chunk g's sums go
  int64_t n, chunk;
  int C_in, C_out;
  hipStream_t st;
};
// A workgroup's tile of dw and its rows.
struct WeightJob {
  int64_t job, begin, end;
  int c0, n0;
};
template <int BC, int BN> __device__ __forceinline__ WeightJob weight_job(const LinearWeight& a) {
  const int64_t nc = (a.C_in + BC - 1) / BC, nn = (a.C_out + BN - 1) / BN;
  const int64_t id = die_order(blockIdx.x, gridDim.x), job = id / (nc * nn);
  const int64_t begin = job * a.chunk, end = begin + a.chunk < a.n ? begin + a.chunk : a.n;
  return WeightJob{job, begin, end, static_cast<int>(id / nn % nc) * BC,
                   static_cast<int>(id % nn) * BN};
}
// The finished tile, straight from the registers (32 bytes of a row by two lanes).
template <int FC, int FN>
__device__ __forceinline__ void store_sums(const f32x16 (&acc)[FN][FC], const LinearWeight& a,
                                           int64_t job, int r0, int c0) {
  const int lane = threadIdx.x & 63;
  float* out = a.dw + job * a.C_in * a.C_out;
#pragma unroll
  for (int n = 0; n < FN; ++n)
#pragma unroll
    for (int m = 0; m < FC; ++m) {
      const int64_t r = r0 + 32 * m + (lane & 31);
      if (r >= a.C_in) continue;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int c = c0 + 32 * n + 8 * q + 4 * (lane >> 5);
        float v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = acc[n][m][4 * q + i];
        if (c < a.C_out) store_left(out + r * a.C_out + c, pack(v), a.C_out - c);
      }
    }
}

// Whole aligned 16-byte pieces: straight to LDS through a ring of three stages of 64 bytes.
// Bound as k_linear: matrix cores 37 % of the busy cycles, LDS 18 (348,208 x 256 x 1024 bf16: 260 us and
// 11 for the chunks' sums, 680 TFLOP/s; 902,504 x 64 x 64: 54, 4.3 TB/s).
template <typename T, int BC, int BN, int WR, int WC>
__global__ __launch_bounds__(64 * WR * WC, 2) void k_linear_dw_ring(LinearWeight a) {
  constexpr int KB = 64, kRing = 3;
  typedef KTile<T, BC, KB> TX;
  typedef KTile<T, BN, KB> TY;
  constexpr int VEC = Row<T>::VEC, BK = kBK<T, KB>, NT = 64 * WR * WC;
  constexpr int FC = BC / WR / 32, FN = BN / WC / 32;
  constexpr int PX = TX::PIECES / NT, PY = TY::PIECES / NT, NP = TX::PIECES + TY::PIECES;
  static_assert(NT / TX::PR % 4 == 0 && NT / TY::PR % 4 == 0 && (sizeof(T) == 2 || (NT / TX::PR % 8 == 0 && NT / TY::PR % 8 == 0)),
                "a lane's pieces of a stage have one place in their rows");
  __shared__ u32x4_t s_buf0[NP], s_buf1[NP], s_buf2[NP];
  const T *const x = static_cast<const T*>(a.x), *const dy = static_cast<const T*>(a.dy);
  const WeightJob t = weight_job<BC, BN>(a);
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int jx = threadIdx.x / TX::PR, jy = threadIdx.x / TY::PR;
  const int cx = t.c0 + (TX::at(jx, threadIdx.x % TX::PR) - jx * TX::PR) * VEC;
  const int cy = t.n0 + (TY::at(jy, threadIdx.x % TY::PR) - jy * TY::PR) * VEC;
  // columns past the last one are read as others: nothing of them is stored
  const T* px = x + (t.begin + jx) * a.C_in + (cx < a.C_in ? cx : 0);
  const T* py = dy + (t.begin + jy) * a.C_out + (cy < a.C_out ? cy : 0);
  const int64_t sx = static_cast<int64_t>(NT / TX::PR) * a.C_in;
  const int64_t sy = static_cast<int64_t>(NT / TY::PR) * a.C_out;
  const T* const zero = reinterpret_cast<const T*>(&g_zeros);
  int64_t rj = t.begin;                            // the next stage to request
  // (stages past the last one are asked for too, as zeros)
  auto request = [&](u32x4_t* buf) {
    const int64_t left = t.end - rj;
#pragma unroll
    for (int i = 0; i < PX; ++i)
      load_to_lds(left >= BK || jx + NT / TX::PR * i < left ? px + sx * i : zero,
                  buf + NT * i + 64 * wave);
#pragma unroll
    for (int i = 0; i < PY; ++i)
      load_to_lds(left >= BK || jy + NT / TY::PR * i < left ? py + sy * i : zero,
                  buf + TX::PIECES + NT * i + 64 * wave);
    rj += BK;
    px += static_cast<int64_t>(BK) * a.C_in;
    py += static_cast<int64_t>(BK) * a.C_out;
  };
  const int wr = wave / WC * (BC / WR), wc = wave % WC * (BN / WC);
  const bool bias = a.db && t.c0 == 0 && wr == 0;  // (uniform over the wave)
  f32x16 acc[FN][FC];
  float sum[FN];
#pragma unroll
  for (int n = 0; n < FN; ++n) {
    sum[n] = 0.0f;
#pragma unroll
    for (int m = 0; m < FC; ++m)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[n][m][i] = 0.0f;
  }
  const typename TX::template Reader<32, FC> x_of(wr, lane);
  const typename TY::template Reader<32, FN> dy_of(wc, lane);
  auto stage = [&](const u32x4_t* buf, u32x4_t* before) {
    stage_barrier<(PX + PY) * (kRing - 2)>();
    request(before);
    multiply_stage<T, KB, FC, FN>(
        acc, [&](int m, int q) { return x_of(buf, m, q); },
        [&](int n, int q) {
          const typename Mma<T>::Frag f = dy_of(buf + TX::PIECES, n, q);
          if (bias) sum[n] = frag_sum(sum[n], f);
          return f;
        });
  };
  const int64_t nk = t.end > t.begin ? (t.end - t.begin + BK - 1) / BK : 0;
  request(s_buf0);
  request(s_buf1);
  for (int64_t s = 0; s < nk; s += kRing) {
    stage(s_buf0, s_buf2);
    if (s + 1 < nk) stage(s_buf1, s_buf0);
    if (s + 2 < nk) stage(s_buf2, s_buf1);
  }
  stage_barrier<0>();                              // (no load to LDS outlives the workgroup)
  if (bias) {
#pragma unroll
    for (int n = 0; n < FN; ++n) {
      const float v = sum[n] + __shfl_xor(sum[n], 32, 64);
      const int col = t.n0 + wc + 32 * n + lane;
      if (lane < 32 && col < a.C_out) a.db[t.job * a.C_out + col] = v;
    }
  }
  store_sums<FC, FN>(acc, a, t.job, t.c0 + wr, t.n0 + wc);
}

// Eight fp32 numbers as three bf16 ones each that add up to them, cut off rather than rounded: 8 bits
// at the top, the 8 behind them, the 8 that are left.  An infinity is its first number, beside
// zeros.  (A NaN's three are NaN.)
template <bool INF>
__device__ __forceinline__ void split_bf16(const float (&v)[8], u32x4_t (&part)[3]) {
  // (the high halves of b and a)
  const auto both = [](float a, float b) {
    return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
  };
  const auto top = [](float a) { return __uint_as_float(__float_as_uint(a) & 0xffff0000u); };
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float a = v[2 * i], b = v[2 * i + 1];
    part[0][i] = both(a, b);
    a = INF && fabsf(a) == INFINITY ? 0.0f : a - top(a);
    b = INF && fabsf(b) == INFINITY ? 0.0f : b - top(b);
    part[1][i] = both(a, b);
    part[2][i] = both(a - top(a), b - top(b));
  }
}

// The same through registers: cut or unaligned pieces, and rows in 8 bits (X8), whose scale goes
// to the other operand: scale * dy, rounded to fp32, enters as three bf16 numbers that are exactly
// it, beside the e4m3 values as the bf16 numbers they are, so that every product is exact
// wherever its factors lie.  (Two f16 numbers under a power of two for the tile: 22 bits of the
// tile's largest and fewer of what is far below it, at two thirds of the products: 16,384 x 2048 x
// 2048 300 us, 348,208 x 256 x 1024 421, and 363 and 509 so.)
// WHOLE: rows are of whole pieces.
// 16,384 x 2048 x 2048 of 8 bits: 349 us and 14 for the sums, 1,180 TFLOP/s of the three products it
// is (a large library product 1,147): matrix cores 60 % of the busy cycles, vector ALU 39, LDS 27.
template <typename T, bool X8, int BC, int BN, int WR, int WC, int KB, bool WHOLE>
__global__ __launch_bounds__(64 * WR * WC, 2) void k_linear_dw(LinearWeight a) {
  typedef KTile<T, BC, KB> TX;
  typedef KTile<T, BN, KB> TY;
  constexpr int VEC = Row<T>::VEC, BK = kBK<T, KB>, NT = 64 * WR * WC;
  constexpr int FC = BC / WR / 32, FN = BN / WC / 32;
  constexpr int PX = TX::PIECES / NT, PY = TY::PIECES / NT, NL = X8 ? 3 : 1;
  __shared__ u32x4_t s_x[TX::PIECES], s_y[NL][TY::PIECES];
  __shared__ float s_db[NT / TY::PR][BN];
  const T* const dy = static_cast<const T*>(a.dy);
  const WeightJob t = weight_job<BC, BN>(a);
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int jx = threadIdx.x / TX::PR, px = threadIdx.x % TX::PR;
  const int jy = threadIdx.x / TY::PR, py = threadIdx.x % TY::PR;
  const int cx = t.c0 + px * VEC, cy = t.n0 + py * VEC;
  uint2 rx8[PX];
  u32x4_t rx[PX], ry[PY];
  float rs[PY];
  auto request = [&](int64_t j0) {
#pragma unroll
    for (int i = 0; i < PX; ++i) {
      const int64_t j = j0 + jx + NT / TX::PR * i;
      const int left = j < t.end ? a.C_in - cx : 0;
      if constexpr (X8) {
        const uint8_t* p = static_cast<const uint8_t*>(a.x) + j * a.C_in + cx;
        if constexpr (WHOLE)
          __builtin_memcpy(&rx8[i], left > 0 ? p : reinterpret_cast<const uint8_t*>(&g_zeros), 8);
        else
          rx8[i] = load8_left(p, left);
      } else {
        rx[i] = load_left<T, WHOLE>(static_cast<const T*>(a.x) + j * a.C_in + cx, left);
      }
    }
#pragma unroll
    for (int i = 0; i < PY; ++i) {
      const int64_t j = j0 + jy + NT / TY::PR * i;
      ry[i] = load_left<T, WHOLE>(dy + j * a.C_out + cy, j < t.end ? a.C_out - cy : 0);
      rs[i] = X8 && j < t.end ? a.x_scale[j] : 0.0f;
    }
  };
  const bool bias = a.db && t.c0 == 0;             // (uniform)
  float sum[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) sum[e] = 0.0f;
  f32x16 acc[FN][FC];
#pragma unroll
  for (int n = 0; n < FN; ++n)
#pragma unroll
    for (int m = 0; m < FC; ++m)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[n][m][i] = 0.0f;
  const int wr = wave / WC * (BC / WR), wc = wave % WC * (BN / WC);
  const typename TX::template Reader<32, FC> x_of(wr, lane);
  const typename TY::template Reader<32, FN> dy_of(wc, lane);
  if (t.begin < t.end) request(t.begin);
  for (int64_t j0 = t.begin; j0 < t.end; j0 += BK) {
    if (bias) {
#pragma unroll
      for (int i = 0; i < PY; ++i) {
        float u[VEC];
        unpack(ry[i], u);
#pragma unroll
        for (int e = 0; e < VEC; ++e) sum[e] += u[e];
      }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < PX; ++i)
      s_x[TX::at(jx + NT / TX::PR * i, px)] = X8 ? widen(rx8[i].x, rx8[i].y) : rx[i];
#pragma unroll
    for (int i = 0; i < PY; ++i) {
      const int to = TY::at(jy + NT / TY::PR * i, py);
      if constexpr (X8) {
        float v[VEC], most = 0.0f;
        unpack(ry[i], v);
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          v[e] *= rs[i];
          most = fmaxf(most, fabsf(v[e]));
        }
        u32x4_t part[3];
        if (most < INFINITY) split_bf16<false>(v, part);
        else split_bf16<true>(v, part);
#pragma unroll
        for (int l = 0; l < NL; ++l) s_y[l][to] = part[l];
      } else {
        s_y[0][to] = ry[i];
      }
    }
    __syncthreads();
    if (j0 + BK < t.end) request(j0 + BK);
    if constexpr (X8) {
#pragma unroll
      for (int q = 0; q < BK / 16; ++q) {
        bf16x8 fx[FC], fy[NL][FN];
#pragma unroll
        for (int m = 0; m < FC; ++m) fx[m] = x_of(s_x, m, q);
#pragma unroll
        for (int l = 0; l < NL; ++l)
#pragma unroll
          for (int n = 0; n < FN; ++n) fy[l][n] = dy_of(s_y[l], n, q);
#pragma unroll
        for (int l = 0; l < NL; ++l)
#pragma unroll
          for (int n = 0; n < FN; ++n)
#pragma unroll
            for (int m = 0; m < FC; ++m) acc[n][m] = Mma<T>::mma(fy[l][n], fx[m], acc[n][m]);
        __builtin_amdgcn_sched_barrier(0);
      }
    } else {
      multiply_stage<T, KB, FC, FN>(
          acc, [&](int m, int q) { return x_of(s_x, m, q); },
          [&](int n, int q) { return dy_of(s_y[0], n, q); });
    }
  }
  if (bias) {
#pragma unroll
    for (int e = 0; e < VEC; ++e) s_db[jy][py * VEC + e] = sum[e];
    __syncthreads();
    if (threadIdx.x < BN && t.n0 + static_cast<int>(threadIdx.x) < a.C_out) {
      float s = 0.0f;
#pragma unroll
      for (int q = 0; q < NT / TY::PR; ++q) s += s_db[q][threadIdx.x];
      a.db[t.job * a.C_out + t.n0 + threadIdx.x] = s;
    }
  }
  store_sums<FC, FN>(acc, a, t.job, t.c0 + wr, t.n0 + wc);
}

// The chunks' sums: kThreads / RUNS lanes side by side with four values each, RUNS of them down
// the chunks, every RUNS-th one each, then those in order.  Values are dw's, then db's (from a
// multiple of four on).
template <int RUNS>
__global__ __launch_bounds__(kThreads) void k_linear_sum(const float* __restrict__ part,
                                                         const float* __restrict__ part_db,
                                                         int64_t jobs, int64_t per, int C_out,
                                                         float* __restrict__ dw,
                                                         float* __restrict__ db) {
  constexpr int kLanes = kThreads / RUNS;
  __shared__ f32x4_t s_sum[RUNS][kLanes];
  const int lane = threadIdx.x % kLanes, run = threadIdx.x / kLanes;
  int64_t i = (static_cast<int64_t>(blockIdx.x) * kLanes + lane) * 4, width = per;
  const int64_t whole = (per + 3) / 4 * 4;
  if (i >= whole) {
    i -= whole;
    width = db ? C_out : 0;
    part = part_db;
    dw = db;
  }
  f32x4_t s = {0.0f, 0.0f, 0.0f, 0.0f};
  if (i + 4 <= width) {
#pragma unroll 4
    for (int64_t c = run; c < jobs; c += RUNS)
      s += __builtin_bit_cast(f32x4_t, load_piece(part + c * width + i));
  } else {
    for (int64_t c = run; c < jobs; c += RUNS)
      for (int q = 0; q < 4 && i + q < width; ++q) s[q] += part[c * width + i + q];
  }
  if constexpr (RUNS > 1) {
    s_sum[run][lane] = s;
    __syncthreads();
  }
  if (run == 0 && i < width) {
#pragma unroll
    for (int q = 1; q < RUNS; ++q) s += s_sum[q][lane];
    store_left(dw + i, __builtin_bit_cast(u32x4_t, s), width - i);
  }
}

template <int BM, int BN> bool grid_of(const LinearArgs& a, int threads, uint32_t* blocks) {
  const int64_t n = (a.n + BM - 1) / BM * ((a.cols + BN - 1) / BN);
  *blocks = static_cast<uint32_t>(n);
  return grid_fits(n, threads);
}
template <typename T, typename TO, bool X8, bool BT, int BM, int BN>
int run_any(const LinearArgs& a) {
  uint32_t blocks;
  if (!grid_of<BM, BN>(a, kThreads, &blocks)) return SPCONV_EINVAL;
  k_linear_any<T, TO, X8, BT, BM, BN><<<blocks, kThreads, 0, a.st>>>(a);
  return launched();
}
template <typename T, typename TO, bool X8, bool BT, int BM, int BN, int WR, int WC>
int run_tiles(LinearArgs a) {
  constexpr int NT = 64 * WR * WC;
  uint32_t blocks;
  // (348,208 x 256 -> 1024, its rows in no cache: 531 us, and 468 touched; 1024 -> 256, whose rows the
  // L2 cannot hold: 261, and 308)
  const double row = static_cast<double>(a.red) * (X8 ? 1 : sizeof(T));
  a.touch = BM * row * kResident<BM> / ((a.cols + BN - 1) / BN) <= 4.3e6;
  if (!grid_of<BM, BN>(a, NT, &blocks)) return SPCONV_EINVAL;
  if (linear_past(a.n, a.cols, (a.z ? 2 : 1) * static_cast<int>(sizeof(TO))))
    k_linear<T, TO, X8, BT, BM, BN, WR, WC, true, 1><<<blocks, NT, 0, a.st>>>(a);
  else
    k_linear<T, TO, X8, BT, BM, BN, WR, WC, false, 1><<<blocks, NT, 0, a.st>>>(a);
  return launched();
}
template <typename T, typename TO, bool X8, bool BT> int run_split(const LinearArgs& a) {
  uint32_t blocks;
  if (!grid_of<32, 32>(a, 64 * kSplit, &blocks)) return SPCONV_EINVAL;
  k_linear<T, TO, X8, BT, 32, 32, 1, 1, false, kSplit><<<blocks, 64 * kSplit, 0, a.st>>>(a);
  return launched();
}
template <bool BT, int NK, bool RES> int run_short_of(const LinearArgs& a) {
  // as many workgroups as fit
  const int groups = (a.cols + 255) / 256, slots = (NK == 2 && !RES ? 512 : 256) / groups;
  const int64_t tiles = (a.n + 63) / 64, most = slots > 1 ? slots : 1;
  const int strips = static_cast<int>(tiles < most ? tiles : most);
  if (linear_past(a.n, a.cols, a.z ? 4 : 2))
    k_linear_short<BT, NK, true, RES><<<strips * groups, 512, 0, a.st>>>(a, strips);
  else
    k_linear_short<BT, NK, false, RES><<<strips * groups, 512, 0, a.st>>>(a, strips);
  return launched();
}
template <bool BT, int NK> int run_short(const LinearArgs& a) {
  if constexpr (!BT)
    if (a.side) return run_short_of<BT, NK, true>(a);
  return run_short_of<BT, NK, false>(a);
}
// The kernel that linear_plan says, or k_linear_short where linear_short has a place for it.
template <typename T, typename TO, bool X8, bool BT> int by_size(const LinearArgs& a) {
  const bool whole = (X8 ? a.red % 16 == 0 && aligned_to(a.x, 16) : whole_rows<T>(a.x, a.red)) &&
                     whole_rows<T>(a.w, BT ? a.red : a.cols);
  const LinearPlan p = linear_plan(sizeof(T) == 4 ? SPCONV_F32 : SPCONV_BF16, BT, a.n, a.red,
                                   a.cols, whole);
  if constexpr (sizeof(T) == 4) {
    if (p.kernel == LinearKernel::kFew) {
      uint32_t blocks;
      if constexpr (BT) {
        if (!grid_of<kFewRows, 8>(a, kThreads, &blocks)) return SPCONV_EINVAL;
        k_linear_few_back<TO><<<blocks, kThreads, 0, a.st>>>(a);
      } else {
        if (!grid_of<kFewRows, 16>(a, kFewThreads, &blocks)) return SPCONV_EINVAL;
        k_linear_few<TO><<<blocks, kFewThreads, 0, a.st>>>(a);
      }
      return launched();
    }
  }
  if (p.kernel == LinearKernel::kAny)
    return p.tile == 64 ? run_any<T, TO, X8, BT, 64, 64>(a) : run_any<T, TO, X8, BT, 128, 128>(a);
  if constexpr (sizeof(T) == 2) {
    if constexpr (!X8 && sizeof(TO) == 2) {
      switch (whole && !(BT && a.side) ? linear_short(a.n, a.red, a.cols, a.side) : 0) {
        case 2: return run_short<BT, 2>(a);
        case 4: return run_short<BT, 4>(a);
        case 6: return run_short<BT, 6>(a);
        case 8: return run_short<BT, 8>(a);
      }
    }
    if (p.tile == 256) return run_tiles<T, TO, X8, BT, 256, 128, 4, 2>(a);
  }
  if (p.tile == 128) return run_tiles<T, TO, X8, BT, 128, 128, 2, 2>(a);
  if (p.kernel == LinearKernel::kSplit) return run_split<T, TO, X8, BT>(a);
  return run_tiles<T, TO, X8, BT, 64, 64, 2, 2>(a);
}

// The kernel of exactly the plan's tile (its workgroups are counted for that one): the ring for
// whole aligned pieces of bf16 and fp32, else k_linear_dw.  (bf16 in cut pieces, us in tiles of up
// to 256 and of up to 128: 100,000 x 1001 x 1001 651 and 923, 348,208 x 255 x 1023 696 and 1,030,
// 100,000 x 131 x 300 72 and 77, 485,480 x 174 x 96 133 and 124, 60,000 x 203 x 201 58 and 45.)
template <typename T, bool X8, int BC, int BN, int WR, int KB>
void run_dw_tile(const LinearWeight& a, const DwPlan& p) {
  const uint32_t blocks = static_cast<uint32_t>(p.jobs * p.tiles);
  const bool wx = X8 ? a.C_in % 8 == 0 : whole_rows<T>(a.x, a.C_in);
  const bool whole = wx && whole_rows<T>(a.dy, a.C_out);
  if (!whole)
    k_linear_dw<T, X8, BC, BN, 2, 2, KB, false><<<blocks, 256, 0, a.st>>>(a);
  else if constexpr (X8)
    k_linear_dw<T, X8, BC, BN, 2, 2, KB, true><<<blocks, 256, 0, a.st>>>(a);
  else
    k_linear_dw_ring<T, BC, BN, WR, 2><<<blocks, 128 * WR, 0, a.st>>>(a);
}
template <typename T, bool X8> int run_dw(const LinearWeight& a, const DwPlan& p) {
  switch (p.tile) {
    case 64: run_dw_tile<T, X8, 64, 64, 2, 128>(a, p); break;
    case 128: run_dw_tile<T, X8, 128, 128, 2, 128>(a, p); break;
    case 256:
      if constexpr (sizeof(T) == 2) {
        run_dw_tile<T, X8, 256, 128, 4, 64>(a, p);
        break;
      }
    default: return SPCONV_EINVAL;
  }
  return launched();
}

bool linear_sizes_ok(int64_t n, int C_in, int C_out) {
  return rows_ok(n) && C_in >= 1 && C_out >= 1 && C_in <= (1 << 23) && C_out <= (1 << 23) &&
         static_cast<int64_t>(C_in) * C_out < 0x80000000ll;
}
// A type of rows: `dt` or 8 bits with its scales.
bool rows_type_ok(int dt, const float* scale, int64_t n) {
  return dt == SPCONV_E4M3 ? ptr_ok(scale, n, 4) : dtype_ok(dt) && !scale;
}
size_t row_bytes(int dt) { return dt == SPCONV_E4M3 ? 1 : elem_bytes(dt); }

}  // namespace
}  // namespace spc

using namespace spc;

extern "C" int spconv_linear_forward(int in_dt, const void* x, const float* x_scale, const void* w,
                                     const float* bias, int act, const void* residual, int out_dt,
                                     void* y, void* z, int64_t n, int C_in, int C_out,
                                     void* stream) {
  if (!rows_type_ok(in_dt, x_scale, n) || !dtype_ok(out_dt) || !act_ok(act) ||
      !linear_sizes_ok(n, C_in, C_out))
    return SPCONV_EINVAL;
  const size_t o = elem_bytes(out_dt);
  if (!ptr_ok(x, n, row_bytes(in_dt)) || !ptr_ok(w, 1, in_dt == SPCONV_F32 ? 4 : 2) ||
      !aligned_to(bias, 4) || !aligned_to(residual, o) || !ptr_ok(y, n, o) || !aligned_to(z, o))
    return SPCONV_EINVAL;
  if (n == 0) return SPCONV_OK;
  const LinearArgs a{x, x_scale, w, bias, act, residual, nullptr, y, z, n, C_in, C_out,
                     static_cast<hipStream_t>(stream)};
  const bool wide = out_dt == SPCONV_F32;
  if (in_dt == SPCONV_F32)
    return wide ? by_size<float, float, false, false>(a) : by_size<float, bf16_t, false, false>(a);
  if (in_dt == SPCONV_BF16)
    return wide ? by_size<bf16_t, float, false, false>(a) : by_size<bf16_t, bf16_t, false, false>(a);
  return wide ? by_size<bf16_t, float, true, false>(a) : by_size<bf16_t, bf16_t, true, false>(a);
}

extern "C" int spconv_linear_backward_data(int dt, const void* dy, const void* w, int act,
                                           int pre_dt, const void* pre, const float* pre_scale,
                                           int out_dt, void* dx, int64_t n, int C_in, int C_out,
                                           void* stream) {
  if (!dtype_ok(dt) || !dtype_ok(out_dt) || !act_ok(act) || !linear_sizes_ok(n, C_in, C_out) ||
      (pre_dt != out_dt && pre_dt != SPCONV_E4M3) ||
      (act == SPCONV_ACT_NONE ? pre || pre_scale : !rows_type_ok(pre_dt, pre_scale, n)))
    return SPCONV_EINVAL;
  const size_t e = elem_bytes(dt), o = elem_bytes(out_dt);
  if (!ptr_ok(dy, n, e) || !ptr_ok(w, 1, e) || !ptr_ok(dx, n, o) ||
      (act != SPCONV_ACT_NONE && !ptr_ok(pre, n, row_bytes(pre_dt))))
    return SPCONV_EINVAL;
  if (n == 0) return SPCONV_OK;
  const LinearArgs a{dy, nullptr, w, nullptr, act, pre, pre_scale, dx, nullptr, n, C_out, C_in,
                     static_cast<hipStream_t>(stream)};
  const bool wide = out_dt == SPCONV_F32;
  if (dt == SPCONV_F32)
    return wide ? by_size<float, float, false, true>(a) : by_size<float, bf16_t, false, true>(a);
  return wide ? by_size<bf16_t, float, false, true>(a) : by_size<bf16_t, bf16_t, false, true>(a);
}

extern "C" int spconv_linear_backward_weight_workspace(int x_dt, int64_t n, int C_in, int C_out,
                                                       size_t* bytes) {
  if ((!dtype_ok(x_dt) && x_dt != SPCONV_E4M3) || !linear_sizes_ok(n, C_in, C_out) || !bytes)
    return SPCONV_EINVAL;
  *bytes = linear_dw_plan(x_dt, n, C_in, C_out).bytes;
  return SPCONV_OK;
}

extern "C" int spconv_linear_backward_weight(int x_dt, const void* x, const float* x_scale,
                                             const void* dy, float* dw, float* db, int64_t n,
                                             int C_in, int C_out, void* workspace,
                                             size_t workspace_bytes, void* stream) {
  if (!rows_type_ok(x_dt, x_scale, n) || !linear_sizes_ok(n, C_in, C_out)) return SPCONV_EINVAL;
  const DwPlan plan = linear_dw_plan(x_dt, n, C_in, C_out);
  if (!ptr_ok(x, n, row_bytes(x_dt)) || !ptr_ok(dy, n, x_dt == SPCONV_F32 ? 4 : 2) ||
      !ptr_ok(dw, 1, 4) || !aligned_to(db, 4) ||
      (plan.bytes && (!workspace || !aligned_to(workspace, 16) || workspace_bytes < plan.bytes)))
    return SPCONV_EINVAL;
  if (!grid_fits(plan.jobs * plan.tiles, kThreads)) return SPCONV_EINVAL;
  hipStream_t st = static_cast<hipStream_t>(stream);
  const int64_t per = static_cast<int64_t>(C_in) * C_out;
  LinearWeight a{x, x_scale, dy, dw, db, n, plan.chunk, C_in, C_out, st};
  if (plan.jobs > 1) {
    a.dw = static_cast<float*>(workspace);
    a.db = db ? a.dw + plan.jobs * per : nullptr;
  }
  const int status = x_dt == SPCONV_E4M3   ? run_dw<bf16_t, true>(a, plan)
                     : x_dt == SPCONV_BF16 ? run_dw<bf16_t, false>(a, plan)
                                           : run_dw<float, false>(a, plan);
  if (status != SPCONV_OK) return status;
  if (plan.jobs > 1) {
    const int64_t values = (per + 3) / 4 * 4 + (db ? C_out : 0);
    if (dw_sum_runs(plan, 1, values) == 8)
      k_linear_sum<8><<<static_cast<uint32_t>((values + kThreads / 2 - 1) / (kThreads / 2)),
                        kThreads, 0, st>>>(a.dw, a.db, plan.jobs, per, C_out, dw, db);
    else
      k_linear_sum<1><<<static_cast<uint32_t>((values + 4 * kThreads - 1) / (4 * kThreads)),
                        kThreads, 0, st>>>(a.dw, a.db, plan.jobs, per, C_out, dw, db);
  }
  return launched();
}
