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

// Staged tiles in LDS, in 16-byte pieces.
//
// RTile: R rows of 128 bytes of the reduction.  A fragment read takes one piece
// column of 16 rows per cycle, so pieces are permuted by the row's bits 1 to 3:
// 16 rows then cover the 64 banks once.
template <typename T, int R> struct RTile {
  static constexpr int VEC = Row<T>::VEC, BK = 128 / static_cast<int>(sizeof(T));
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
  static constexpr int VEC = Row<T>::VEC, BK = 128 / static_cast<int>(sizeof(T));
  static constexpr int PR = W / VEC;                // pieces per row
  static constexpr int PIECES = BK * PR, BYTES = PIECES * 16;
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

// A piece of a row: `left` elements of it remain (<= 0: none, zeros).
// WHOLE: remaining counts are multiples of a piece.
template <typename T, bool WHOLE>
__device__ __forceinline__ u32x4_t load_left(const T* p, int64_t left) {
  constexpr int VEC = Row<T>::VEC;
  u32x4_t v = {0u, 0u, 0u, 0u};
  if (WHOLE ? left > 0 : left >= VEC) {
    v = load_piece(p);
  } else if (!WHOLE && left > 0) {
    T e[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) e[i] = i < left ? p[i] : T(0);
    __builtin_memcpy(&v, e, 16);
  }
  return v;
}

// Finished fp32 values [BR][BC] of the workgroup go through LDS, rounded to TO,
// so that whole rows leave in 16-byte pieces.  FR x FC blocks of 32 x 32 per
// wave at (r0, c0); acc[fc][fr] as Mma leaves them with the columns as the first
// operand.
template <typename TO, int BR, int BC, int FR, int FC>
__device__ __forceinline__ void tile_to_lds(TO* s, const f32x16 (&acc)[FC][FR], int r0, int c0,
                                            const float* __restrict__ bias, int64_t bias_left,
                                            int relu) {
  constexpr int VO = Row<TO>::VEC, PR = BC / VO;
  const int lane = threadIdx.x & 63, h = lane >> 5;
#pragma unroll
  for (int fc = 0; fc < FC; ++fc)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int c = c0 + 32 * fc + 8 * q + 4 * h;
      float b[4] = {0.0f, 0.0f, 0.0f, 0.0f};
      if (bias) {
#pragma unroll
        for (int i = 0; i < 4; ++i) b[i] = c + i < bias_left ? bias[c + i] : 0.0f;
      }
#pragma unroll
      for (int fr = 0; fr < FR; ++fr) {
        const int r = r0 + 32 * fr + (lane & 31);
        TO v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float z = acc[fc][fr][4 * q + i] + b[i];
          if (relu && z < 0.0f) z = 0.0f;
          v[i] = Row<TO>::put(z);
        }
        const int piece = (c / VO) ^ (r & (PR - 1));
        __builtin_memcpy(__builtin_assume_aligned(s + (r * PR + piece) * VO + c % VO,
                                                  4 * sizeof(TO)),
                         v, sizeof v);
      }
    }
}
template <typename TO, int BR, int BC>
__device__ __forceinline__ u32x4_t lds_piece(const TO* s, int r, int piece) {
  constexpr int VO = Row<TO>::VEC, PR = BC / VO;
  return reinterpret_cast<const u32x4_t*>(s)[r * PR + (piece ^ (r & (PR - 1)))];
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
  hipStream_t st;
};

// Rows x weights of a BM x BN tile: BT false: w[e] is [red][cols] (the forward),
// BT true: w[e] is [cols][red] (the input gradient).  Four waves in 2 x 2.  The
// pieces of the next 128 bytes of the reduction are requested into registers
// while the present ones, in LDS, are multiplied; two LDS buffers, one barrier a
// step.
template <typename T, typename TO, bool BT, int BM, int BN, bool WHOLE>
__global__ __launch_bounds__(kThreads, 2) void k_grouped(GroupedArgs a) {
  typedef Mma<T> M;
  typedef RTile<T, BM> TA;
  typedef RTile<T, BN> TBr;
  typedef KTile<T, BN> TBk;
  constexpr int VEC = Row<T>::VEC, BK = TA::BK, STEPS = BK / M::KS;
  constexpr int FM = BM / 64, FN = BN / 64;
  constexpr int PA = TA::PIECES / kThreads;
  constexpr int PB = TBk::PIECES / kThreads;       // (as many as TBr's)
  constexpr int kStage = TA::BYTES + TBk::BYTES;
  constexpr int kOut = BM * BN * static_cast<int>(sizeof(TO));
  __shared__ __attribute__((aligned(16))) unsigned char
      s_buf[2 * kStage > kOut ? 2 * kStage : kOut];
  const T* const x = static_cast<const T*>(a.x);
  TO* const y = static_cast<TO*>(a.y);
  const int64_t ncol = (a.cols + BN - 1) / BN;
  const int64_t id = die_order(blockIdx.x, gridDim.x);
  const Tile t = find_tile<true>(a.offsets, a.E, a.m, BM, id / ncol);
  if (t.group < 0) return;
  const int64_t n0 = id % ncol * BN;
  const int nrow = static_cast<int>(t.end - t.begin);
  if (t.group == a.E) {                            // behind the last group
    for (int p = threadIdx.x; p < nrow * BN; p += kThreads) {
      const int64_t c = n0 + p % BN;
      if (c < a.cols) y[(t.begin + p / BN) * a.cols + c] = Row<TO>::put(0.0f);
    }
    return;
  }
  const T* const w = static_cast<const T*>(a.w) + static_cast<int64_t>(t.group) * a.red * a.cols;

  // what this lane stages
  const T* pa[PA];
  bool oka[PA];
#pragma unroll
  for (int i = 0; i < PA; ++i) {
    const int r = (threadIdx.x >> 3) + 32 * i;
    int64_t src = -1;
    if (r < nrow) {
      src = a.rows ? a.rows[t.begin + r] : t.begin + r;
      if (src >= a.n_x) src = -1;
    }
    oka[i] = src >= 0;
    pa[i] = x + (src < 0 ? 0 : src) * a.red;
  }
  const int ka = (threadIdx.x & 7) * VEC;
  u32x4_t ra[PA], rb[PB];
  auto request = [&](int64_t k0) {
#pragma unroll
    for (int i = 0; i < PA; ++i)
      ra[i] = load_left<T, WHOLE>(pa[i] + k0 + ka, oka[i] ? a.red - k0 - ka : 0);
#pragma unroll
    for (int i = 0; i < PB; ++i) {
      if constexpr (BT) {
        const int64_t n = n0 + (threadIdx.x >> 3) + 32 * i;
        rb[i] = load_left<T, WHOLE>(w + n * a.red + k0 + ka, n < a.cols ? a.red - k0 - ka : 0);
      } else {
        const int p = threadIdx.x + kThreads * i;
        const int64_t k = k0 + p / TBk::PR, n = n0 + p % TBk::PR * VEC;
        rb[i] = load_left<T, WHOLE>(w + k * a.cols + n, k < a.red ? a.cols - n : 0);
      }
    }
  };
  auto put = [&](int buf) {
    u32x4_t* sa = reinterpret_cast<u32x4_t*>(s_buf + buf * kStage);
    u32x4_t* sb = reinterpret_cast<u32x4_t*>(s_buf + buf * kStage + TA::BYTES);
#pragma unroll
    for (int i = 0; i < PA; ++i)
      sa[TA::at((threadIdx.x >> 3) + 32 * i, threadIdx.x & 7)] = ra[i];
#pragma unroll
    for (int i = 0; i < PB; ++i) {
      if constexpr (BT) {
        sb[TBr::at((threadIdx.x >> 3) + 32 * i, threadIdx.x & 7)] = rb[i];
      } else {
        const int p = threadIdx.x + kThreads * i;
        sb[TBk::at(p / TBk::PR, p % TBk::PR)] = rb[i];
      }
    }
  };

  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int wr = (wave >> 1) * (BM / 2), wc = (wave & 1) * (BN / 2);
  f32x16 acc[FN][FM];
#pragma unroll
  for (int n = 0; n < FN; ++n)
#pragma unroll
    for (int m = 0; m < FM; ++m)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[n][m][i] = 0.0f;

  const int64_t nk = (a.red + BK - 1ll) / BK;
  request(0);
  for (int64_t k = 0; k < nk; ++k) {
    const int buf = static_cast<int>(k & 1);
    put(buf);
    __syncthreads();
    if (k + 1 < nk) request((k + 1) * BK);
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
  }
  __syncthreads();
  TO* so = reinterpret_cast<TO*>(s_buf);
  const float* bias = a.bias ? a.bias + static_cast<int64_t>(t.group) * a.cols + n0 : nullptr;
  tile_to_lds<TO, BM, BN, FM, FN>(so, acc, wr, wc, bias, a.cols - n0, a.relu);
  __syncthreads();
  constexpr int VO = Row<TO>::VEC, PO = BN / VO;
  for (int p = threadIdx.x; p < BM * PO; p += kThreads) {
    const int r = p / PO, piece = p % PO;
    const int64_t left = a.cols - n0 - piece * VO;
    if (r >= nrow || left <= 0) continue;
    const int64_t at = (t.begin + r) * a.cols + n0 + piece * VO;
    u32x4_t v = lds_piece<TO, BM, BN>(so, r, piece);
    if (a.mask) {
      float f[VO], g[VO];
      unpack(v, f);
      unpack(load_left<TO, false>(static_cast<const TO*>(a.mask) + at, left), g);
#pragma unroll
      for (int i = 0; i < VO; ++i) f[i] = g[i] <= 0.0f ? 0.0f : f[i];
      v = pack(f);
    }
    store_left(y + at, v, left);
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
  constexpr int VEC = Row<T>::VEC, BK = TX::BK, STEPS = BK / M::KS;
  constexpr int FC = BC / 64, FN = BN / 64;
  constexpr int PX = TX::PIECES / kThreads, PY = TY::PIECES / kThreads;
  constexpr int kStage = TX::BYTES + TY::BYTES, kOut = BC * BN * 4;
  __shared__ __attribute__((aligned(16))) unsigned char
      s_buf[2 * kStage > kOut ? 2 * kStage : kOut];
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
  u32x4_t rx[PX], ry[PY];
  auto request = [&](int64_t j0) {
#pragma unroll
    for (int i = 0; i < PX; ++i) {
      const int p = threadIdx.x + kThreads * i;
      const int64_t j = j0 + p / TX::PR, c = c0 + p % TX::PR * VEC;
      int64_t src = -1;
      if (j < t.end) {
        src = a.rows ? a.rows[j] : j;
        if (src >= a.n_x) src = -1;
      }
      rx[i] = load_left<T, WHOLE>(x + (src < 0 ? 0 : src) * a.C_in + c,
                                  src >= 0 ? a.C_in - c : 0);
    }
#pragma unroll
    for (int i = 0; i < PY; ++i) {
      const int p = threadIdx.x + kThreads * i;
      const int64_t j = j0 + p / TY::PR, n = n0 + p % TY::PR * VEC;
      ry[i] = load_left<T, WHOLE>(dy + j * a.C_out + n, j < t.end ? a.C_out - n : 0);
    }
  };
  auto put = [&](int buf) {
    u32x4_t* sx = reinterpret_cast<u32x4_t*>(s_buf + buf * kStage);
    u32x4_t* sy = reinterpret_cast<u32x4_t*>(s_buf + buf * kStage + TX::BYTES);
#pragma unroll
    for (int i = 0; i < PX; ++i) {
      const int p = threadIdx.x + kThreads * i;
      sx[TX::at(p / TX::PR, p % TX::PR)] = rx[i];
    }
#pragma unroll
    for (int i = 0; i < PY; ++i) {
      const int p = threadIdx.x + kThreads * i;
      sy[TY::at(p / TY::PR, p % TY::PR)] = ry[i];
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
  if (nk) request(t.begin);
  for (int64_t k = 0; k < nk; ++k) {
    const int buf = static_cast<int>(k & 1);
    put(buf);
    __syncthreads();
    if (k + 1 < nk) request(t.begin + (k + 1) * BK);
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
  __syncthreads();
  float* so = reinterpret_cast<float*>(s_buf);
  tile_to_lds<float, BC, BN, FC, FN>(so, acc, wr, wc, nullptr, 0, 0);
  __syncthreads();
  float* out = a.dw + job * a.C_in * a.C_out;
  constexpr int PO = BN / 4;
  for (int p = threadIdx.x; p < BC * PO; p += kThreads) {
    const int r = p / PO, piece = p % PO;
    const int64_t left = a.C_out - n0 - piece * 4;
    if (c0 + r >= a.C_in || left <= 0) continue;
    store_left(out + (c0 + r) * a.C_out + n0 + piece * 4, lds_piece<float, BC, BN>(so, r, piece),
               left);
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

template <typename T, typename TO, bool BT, int BM, int BN> int run_tile(const GroupedArgs& a) {
  const int64_t blocks = tile_bound(a.m, a.E + 1, BM) * ((a.cols + BN - 1) / BN);
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
  return rows_ok(m) && E >= 1 && E <= 65535 && C_in >= 1 && C_out >= 1 && C_in <= (1 << 24) &&
         C_out <= (1 << 24);
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
                                      C_out, static_cast<hipStream_t>(stream)});
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
                                     C_in, static_cast<hipStream_t>(stream)});
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
