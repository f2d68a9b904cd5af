// Dense products of feature rows with bias, activation and residual in their epilogue, and
// their gradients, on the matrix cores: rows in bf16, fp32 or 8 bits with a scale a row.
//
// 8-bit rows are multiplied as the bf16 numbers they are (every e4m3 value is one), and the
// row's scale is taken out of the sum: forwards it is a factor of the finished row, in the
// weight gradient, where the sum runs over the rows, it goes to the other operand, scale *
// dy, which enters as two bf16 numbers (its upper 8 and the next 8 bits: 2^-17 of a factor
// is lost, less than an fp32 sum of as many terms loses).
#include <type_traits>

#include "rows_act.h"
#include "rows_mma.h"
#include "rows_plan.h"

namespace spc {
namespace {

constexpr int kThreads = 256;

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

// The finished tile of a workgroup of WR x WC waves, FM x FN blocks each, leaves through LDS
// as fp32 rows, a row block of every wave at a time: everything behind the product is done
// on fp32 and rounded once, whole rows go to memory, and a lane has the same columns all along
// (its bias stays in registers).  The residual, or the activation's input, is asked for before
// the barrier that its block's sums wait at.
// Forward: z = acc * scale + bias (z is kept if asked for), y = act(z) + residual.
// BT (input gradient): y = acc * act'(side).
template <typename TO, bool X8, bool BT, int BM, int BN, int WR, int WC>
__device__ __forceinline__ void finish_tile(u32x4_t* lds,
                                            const f32x16 (&acc)[BN / WC / 32][BM / WR / 32],
                                            const LinearArgs& a, int64_t row0, int n0) {
  constexpr int FM = BM / WR / 32, FN = BN / WC / 32, VO = Row<TO>::VEC, NT = 64 * WR * WC;
  constexpr int RW = WR * 32, PR = BN / VO, NPC = RW * PR / NT, Q = VO / 4;
  static_assert(NT % PR == 0 && NPC * NT == RW * PR, "a lane's pieces lie in the same columns");
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, h = lane >> 5;
  const int wrow = wave / WC, wcol = wave % WC;
  const int piece = threadIdx.x % PR, col = n0 + piece * VO, left = a.cols - col;
  float bias[VO];
#pragma unroll
  for (int e = 0; e < VO; ++e) bias[e] = 0.0f;
  if (!BT && a.bias) {
#pragma unroll
    for (int e = 0; e < VO; ++e)
      if (e < left) bias[e] = a.bias[col + e];
  }
  const bool side8 = BT && a.side_scale;
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
      live[i] = r < a.n && left > 0;
      at[i] = r * a.cols + col;
      xs[i] = X8 && live[i] ? a.x_scale[r] : 1.0f;
      if (a.side && live[i]) {
        if (side8) {
          const uint2 u = load8_left(static_cast<const uint8_t*>(a.side) + at[i], left < VO ? left : VO);
          g[i][0] = u.x, g[i][1] = u.y;
          xs[i] = a.side_scale[r];
        } else {
          g[i] = load_left<TO, false>(static_cast<const TO*>(a.side) + at[i], left);
        }
      }
    }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < FN; ++n)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        // 4 adjacent columns of one row in every four registers of a lane
        const int c = col_of<WC>(wcol, n) + 8 * q + 4 * h;
        u32x4_t v;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = __float_as_uint(acc[n][m][4 * q + i]);
        lds[out_at<float, BN>(wrow * 32 + (lane & 31), c / 4)] = v;
      }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NPC; ++i) {
      if (!live[i]) continue;
      const int lr = (threadIdx.x + NT * i) / PR;
      float v[VO];
#pragma unroll
      for (int q = 0; q < Q; ++q) {
        const u32x4_t u = lds[out_at<float, BN>(lr, piece * Q + q)];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[4 * q + e] = __uint_as_float(u[e]);
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
            for (int e = 0; e < VO; ++e) v[e] *= slope<decltype(k)::value>(s[e]);
          });
        }
      } else {
#pragma unroll
        for (int e = 0; e < VO; ++e) v[e] = X8 ? v[e] * xs[i] + bias[e] : v[e] + bias[e];
        if (a.z) store_left<TO>(static_cast<TO*>(a.z) + at[i], pack(v), left);
        by_act(a.act, [&](auto k) {
#pragma unroll
          for (int e = 0; e < VO; ++e) v[e] = activate<decltype(k)::value>(v[e]);
        });
        if (a.side) {
          float s[VO];
          unpack(g[i], s);
#pragma unroll
          for (int e = 0; e < VO; ++e) v[e] += s[e];
        }
      }
      store_left<TO>(static_cast<TO*>(a.y) + at[i], pack(v), left);
    }
  }
}

// Rows x weights for any alignment and width: BT false: w is [red][cols] (the forward), BT true:
// w is [cols][red] (the input gradient).  Through registers, 128 x 128 or 64 x 64 by four
// waves in 2 x 2, stages of 128 bytes of the reduction.  X8: rows in 8 bits, widened on their
// way to LDS.
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
  static_assert(NP * 16 >= 64 * BN * 4, "a row block of the finished tile fits");
  __shared__ u32x4_t s_buf[NP];
  const int ncol = (a.cols + BN - 1) / BN;
  const int64_t id = die_order(blockIdx.x, gridDim.x);
  const int64_t row0 = id / ncol * BM;
  const int n0 = static_cast<int>(id % ncol) * BN;
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
  finish_tile<TO, X8, BT, BM, BN, 2, 2>(s_buf, acc, a, row0, n0);
}

// Weight gradient of a BC x BN tile over a chunk of the rows: dw[c][n] = sum_j x[j][c] dy[j][n],
// the rows staged as the reduction, through registers.  Chunk `job` leaves its sums as
// part[job]; the workgroups of the first rows of dw also sum dy.  No atomics: the chunks are
// added in their order.
struct LinearWeight {
  const void* x;
  const float* x_scale;
  const void* dy;
  float *dw, *db;              // where chunk g's sums go
  int64_t n, chunk;
  int C_in, C_out;
  hipStream_t st;
};
template <typename T, bool X8, int BC, int BN>
__global__ __launch_bounds__(kThreads, 2) void k_linear_dw(LinearWeight a) {
  constexpr int KB = 128, WC = 2;
  typedef KTile<T, BC, KB> TX;
  typedef KTile<T, BN, KB> TY;
  constexpr int VEC = Row<T>::VEC, BK = kBK<T, KB>, NT = kThreads;
  constexpr int FC = BC / 64, FN = BN / 64;
  constexpr int PX = TX::PIECES / NT, PY = TY::PIECES / NT, NL = X8 ? 2 : 1;
  __shared__ u32x4_t s_x[TX::PIECES], s_y[NL][TY::PIECES];
  __shared__ float s_db[NT / TY::PR][BN + 1];
  const T* const dy = static_cast<const T*>(a.dy);
  const int64_t nc = (a.C_in + BC - 1) / BC, nn = (a.C_out + BN - 1) / BN;
  const int64_t id = die_order(blockIdx.x, gridDim.x), job = id / (nc * nn);
  const int c0 = static_cast<int>(id / nn % nc) * BC, n0 = static_cast<int>(id % nn) * BN;
  const int64_t begin = job * a.chunk, end = begin + a.chunk < a.n ? begin + a.chunk : a.n;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int jx = threadIdx.x / TX::PR, px = threadIdx.x % TX::PR;
  const int jy = threadIdx.x / TY::PR, py = threadIdx.x % TY::PR;
  const int cx = c0 + px * VEC, cy = n0 + py * VEC;
  u32x4_t rx[PX], ry[PY];
  float rs[PY];
  auto request = [&](int64_t j0) {
#pragma unroll
    for (int i = 0; i < PX; ++i) {
      const int64_t j = j0 + jx + NT / TX::PR * i;
      const int left = j < end ? a.C_in - cx : 0;
      if constexpr (X8) {
        const uint2 u = load8_left(static_cast<const uint8_t*>(a.x) + j * a.C_in + cx, left);
        rx[i] = widen(u.x, u.y);
      } else {
        rx[i] = load_left<T, false>(static_cast<const T*>(a.x) + j * a.C_in + cx, left);
      }
    }
#pragma unroll
    for (int i = 0; i < PY; ++i) {
      const int64_t j = j0 + jy + NT / TY::PR * i;
      ry[i] = load_left<T, false>(dy + j * a.C_out + cy, j < end ? a.C_out - cy : 0);
      rs[i] = X8 && j < end ? a.x_scale[j] : 0.0f;
    }
  };
  const bool bias = a.db && c0 == 0;               // (uniform)
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
  const int wr = wave / WC * (BC / 2), wc = wave % WC * (BN / 2);
  const typename TX::template Reader<32, FC> x_of(wr, lane);
  const typename TY::template Reader<32, FN> dy_of(wc, lane);
  if (begin < end) request(begin);
  for (int64_t j0 = begin; j0 < end; j0 += BK) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < PX; ++i) s_x[TX::at(jx + NT / TX::PR * i, px)] = rx[i];
#pragma unroll
    for (int i = 0; i < PY; ++i) {
      const int to = TY::at(jy + NT / TY::PR * i, py);
      if constexpr (X8) {
        float v[VEC], lo[VEC];
        unpack(ry[i], v);
        if (bias) {
#pragma unroll
          for (int e = 0; e < VEC; ++e) sum[e] += v[e];
        }
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          v[e] *= rs[i];
          const float up = Row<T>::get(Row<T>::put(v[e]));
          // (an infinity or NaN is all in the upper part)
          lo[e] = magnitude(up) < 0x7f800000u ? v[e] - up : 0.0f;
        }
        s_y[0][to] = pack(v);
        s_y[NL - 1][to] = pack(lo);
      } else {
        if (bias) {
          float v[VEC];
          unpack(ry[i], v);
#pragma unroll
          for (int e = 0; e < VEC; ++e) sum[e] += v[e];
        }
        s_y[0][to] = ry[i];
      }
    }
    __syncthreads();
    if (j0 + BK < end) request(j0 + BK);
#pragma unroll
    for (int l = 0; l < NL; ++l)
      multiply_stage<T, KB, FC, FN>(
          acc, [&](int m, int q) { return x_of(s_x, m, q); },
          [&](int n, int q) { return dy_of(s_y[l], n, q); });
  }
  if (bias) {
#pragma unroll
    for (int e = 0; e < VEC; ++e) s_db[jy][py * VEC + e] = sum[e];
    __syncthreads();
    if (threadIdx.x < BN && n0 + static_cast<int>(threadIdx.x) < a.C_out) {
      float s = 0.0f;
#pragma unroll
      for (int q = 0; q < NT / TY::PR; ++q) s += s_db[q][threadIdx.x];
      a.db[job * a.C_out + n0 + threadIdx.x] = s;
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
        const int c = n0 + wc + 32 * n + 8 * q + 4 * (lane >> 5);
        float v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = acc[n][m][4 * q + i];
        if (c < a.C_out) store_left(out + r * a.C_out + c, pack(v), a.C_out - c);
      }
    }
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

template <typename T, typename TO, bool X8, bool BT, int BM, int BN>
int run_any(const LinearArgs& a) {
  const int64_t blocks = (a.n + BM - 1) / BM * ((a.cols + BN - 1) / BN);
  if (!grid_fits(blocks, kThreads)) return SPCONV_EINVAL;
  k_linear_any<T, TO, X8, BT, BM, BN><<<static_cast<uint32_t>(blocks), kThreads, 0, a.st>>>(a);
  return launched();
}
template <typename T, typename TO, bool X8, bool BT> int by_size(const LinearArgs& a) {
  const int64_t tiles = (a.n + 127) / 128 * ((a.cols + 127) / 128);
  if (a.cols <= 64 || tiles < 1024) return run_any<T, TO, X8, BT, 64, 64>(a);
  return run_any<T, TO, X8, BT, 128, 128>(a);
}

// How the weight gradient is cut.
DwPlan weight_plan(int x_dt, int64_t n, int C_in, int C_out) {
  DwPlan p = dw_plan(x_dt == SPCONV_F32 ? SPCONV_F32 : SPCONV_BF16, n, 1, C_in, C_out, false);
  if (!p.chunk) p.chunk = n < 1 ? 1 : n;
  p.jobs = n < 1 ? 1 : (n + p.chunk - 1) / p.chunk;
  p.bytes = p.jobs > 1
                ? static_cast<size_t>(p.jobs) * (static_cast<size_t>(C_in) * C_out + C_out) * 4
                : 0;
  return p;
}
template <typename T, bool X8> void run_dw(const LinearWeight& a, const DwPlan& p) {
  const uint32_t blocks = static_cast<uint32_t>(p.jobs * p.tiles);
  if (p.tile == 128) k_linear_dw<T, X8, 128, 128><<<blocks, kThreads, 0, a.st>>>(a);
  else k_linear_dw<T, X8, 64, 64><<<blocks, kThreads, 0, a.st>>>(a);
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
  *bytes = weight_plan(x_dt, n, C_in, C_out).bytes;
  return SPCONV_OK;
}

extern "C" int spconv_linear_backward_weight(int x_dt, const void* x, const float* x_scale,
                                             const void* dy, float* dw, float* db, int64_t n,
                                             int C_in, int C_out, void* workspace,
                                             size_t workspace_bytes, void* stream) {
  if (!rows_type_ok(x_dt, x_scale, n) || !linear_sizes_ok(n, C_in, C_out)) return SPCONV_EINVAL;
  const DwPlan plan = weight_plan(x_dt, n, C_in, C_out);
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
  if (x_dt == SPCONV_E4M3) run_dw<bf16_t, true>(a, plan);
  else if (x_dt == SPCONV_BF16) run_dw<bf16_t, false>(a, plan);
  else run_dw<float, false>(a, plan);
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
