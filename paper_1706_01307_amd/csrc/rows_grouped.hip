// Products of ragged groups of rows, each group with its own weights, and their
// gradients, on the matrix cores.
//
// Which rows a workgroup has is found on the device: the groups' row tiles are
// numbered in order, and each wave finds the tile's group by a running sum over
// the offsets, 64 groups at a time.  No host knows the group sizes.
#include <type_traits>

#include "rows.h"
#include "rows_plan.h"

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

// The positions [begin, end) of a group.
struct Span {
  int32_t begin, end;
};
__device__ __forceinline__ int32_t clamp_offset(int32_t v, int64_t m) {
  return v < 0 ? 0 : v > m ? static_cast<int32_t>(m) : v;
}
// Those of group e0 + lane, the positions behind the last group as group E
// (WITH_TAIL), none from there on.  Offsets are moved into [0, m], and one below
// those before it counts as the largest of them: whatever they hold, groups do not
// overlap, and so have no more tiles or chunks than a launch and its workspace are
// sized for.  `top` is the largest offset up to e0's, for the next 64 groups then.
// The whole wave calls it; offsets that ascend cost one comparison.
template <bool WITH_TAIL>
__device__ __forceinline__ Span group_span(const int32_t* __restrict__ offsets, int E, int64_t m,
                                           int e0, int32_t* top) {
  const int lane = threadIdx.x & 63, e = e0 + lane;
  Span s{*top, *top};
  if (e < E + (WITH_TAIL ? 1 : 0)) {
    const int32_t a = offsets[e], b = offsets[e < E ? e + 1 : e];   // (both on their way)
    s.begin = clamp_offset(a, m);
    s.end = clamp_offset(e < E ? b : static_cast<int32_t>(m), m);
  }
  if (__ballot(s.begin < *top || s.end < s.begin)) {
    s.begin = s.begin < *top ? *top : s.begin;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const int32_t o = __shfl_up(s.begin, d, 64);
      if (lane >= d && o > s.begin) s.begin = o;
    }
    s.end = s.end < s.begin ? s.begin : s.end;
  }
  *top = __builtin_amdgcn_readlane(s.end, 63);
  return s;
}
// op over the lanes of a wave; all of them get it.
template <typename Op> __device__ __forceinline__ uint32_t wave_reduce(uint32_t v, Op op) {
  v = op(v, lane_other<1>(v));
  v = op(v, lane_other<2>(v));
  v = op(v, lane_other<4>(v));
  v = op(v, lane_other<8>(v));
  const auto p = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  v = op(p[0], p[1]);
  const auto q = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return op(q[0], q[1]);
}
// A lane's part, of NT, of the largest offset up to group e's.
template <int NT>
__device__ __forceinline__ uint32_t part_top(const int32_t* __restrict__ offsets, int64_t m,
                                             int e) {
  uint32_t top = 0;
#pragma unroll 8
  for (int g = threadIdx.x; g <= e; g += NT) {
    const uint32_t o = static_cast<uint32_t>(clamp_offset(offsets[g], m));
    top = o > top ? o : top;
  }
  return top;
}

// Tile t of the groups cut into tiles of BM positions, the positions behind
// the last group as group E (WITH_TAIL).  Every wave of the workgroup calls it
// and gets the same answer.
template <bool WITH_TAIL>
__device__ __forceinline__ Tile find_tile(const int32_t* __restrict__ offsets, int E, int64_t m,
                                          int64_t BM, int64_t t) {
  const int lane = threadIdx.x & 63;
  const int groups = E + (WITH_TAIL ? 1 : 0);
  int64_t before = 0;
  int32_t top = 0;
  for (int e0 = 0; e0 < groups; e0 += 64) {
    const Span s = group_span<WITH_TAIL>(offsets, E, m, e0, &top);
    const int tiles = static_cast<int>((static_cast<int64_t>(s.end) - s.begin + BM - 1) / BM);
    // (the running sum only where the tile is among these groups')
    const bool last = e0 + 64 >= groups;
    const uint32_t all = last ? 0 : wave_reduce(static_cast<uint32_t>(tiles),
                                                [](uint32_t u, uint32_t v) { return u + v; });
    if (last || before + all > t) {
      int sum = tiles;
#pragma unroll
      for (int d = 1; d < 64; d *= 2) {
        const int o = __shfl_up(sum, d, 64);
        if (lane >= d) sum += o;
      }
      const uint64_t hit = __ballot(before + sum > t);
      if (!hit) break;
      const int src = __ffsll(static_cast<unsigned long long>(hit)) - 1;
      Tile r;
      r.group = e0 + src;
      r.index = static_cast<int>(t - before) - __builtin_amdgcn_readlane(sum - tiles, src);
      const int64_t end = __builtin_amdgcn_readlane(s.end, src);
      r.begin = __builtin_amdgcn_readlane(s.begin, src) + static_cast<int64_t>(r.index) * BM;
      r.end = r.begin + BM < end ? r.begin + BM : end;
      return r;
    }
    before += all;
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

// What a workgroup of the products has to do: `nrow` positions from `begin` of a
// group, the columns from n0.
struct Job {
  int group, nrow, n0;
  int64_t begin;
};
// Workgroup -> job, `span` columns each.  False: nothing (or only zeros, written
// here).
template <typename TO, int BM>
__device__ __forceinline__ bool grouped_job(const GroupedArgs& a, int span, Job* j) {
  const int nspan = (a.cols + span - 1) / span;
  const int64_t id = die_order(blockIdx.x, gridDim.x);
  const Tile t = find_tile<true>(a.offsets, a.E, a.m, BM, id / nspan);
  if (t.group < 0) return false;
  j->group = t.group;
  j->begin = t.begin;
  j->nrow = static_cast<int>(t.end - t.begin);
  j->n0 = static_cast<int>(id % nspan) * span;
  if (t.group < a.E) return true;
  // behind the last group
  const int end = a.cols - j->n0 < span ? a.cols : j->n0 + span;
  TO* y = static_cast<TO*>(a.y);
  for (int r = 0; r < j->nrow; ++r)
    for (int c = j->n0 + threadIdx.x; c < end; c += blockDim.x)
      y[(t.begin + r) * a.cols + c] = Row<TO>::put(0.0f);
  return false;
}
// The row that position `begin + r` reads, -1 for a row of zeros.
__device__ __forceinline__ int64_t source_row(const GroupedArgs& a, const Job& j, int r) {
  if (r >= j.nrow) return -1;
  const int64_t src = a.rows ? a.rows[j.begin + r] : j.begin + r;
  return src < a.n_x ? src : -1;
}

// The bias of columns n0 .. n0 + N, zeros without one, in LDS before a tile is
// finished (a load then would wait for every load in flight).
template <int N>
__device__ __forceinline__ void load_bias(const GroupedArgs& a, const Job& j, int n0,
                                          float* s_bias) {
  const float* b = a.bias ? a.bias + static_cast<int64_t>(j.group) * a.cols : nullptr;
  for (int c = threadIdx.x; c < N; c += blockDim.x)
    s_bias[c] = b && n0 + c < a.cols ? b[n0 + c] : 0.0f;
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

// The finished tile of a workgroup of WR x WC waves, FM x FN blocks each, leaves
// through LDS as whole rows, in parts that fit `lds` (BYTES) and are up to four
// pieces a lane: FNP column and FMP row blocks of every wave at a time.  A barrier
// before and within each part; its mask (MASK) is asked for while the part before is
// finished (65,536 x 512 -> 2048 bf16, backwards: 261 us; when a part needs it, 314),
// unless the last pieces of its rows may be cut (WHOLE false): those loads wait for
// one another.
template <typename TO, bool MASK, bool WHOLE, bool RELU, int BM, int BN, int WR, int WC,
          int BYTES>
__device__ __forceinline__ void store_tile_rows(
    u32x4_t* lds, const f32x16 (&acc)[BN / WC / 32][BM / WR / 32], const float* s_bias,
    const GroupedArgs& a, const Job& j, int n0) {
  constexpr int FM = BM / WR / 32, FN = BN / WC / 32, VO = Row<TO>::VEC;
  constexpr int TOB = static_cast<int>(sizeof(TO));
  constexpr int NT = 64 * WR * WC, ROOM = BYTES < 64 * NT ? BYTES : 64 * NT;
  constexpr int FNP = BM * BN * TOB <= ROOM ? FN : 1;
  constexpr int CW = WC * 32 * FNP;                // columns of a part
  constexpr int FMP = BM * CW * TOB <= ROOM ? FM : BM * CW * TOB <= 2 * ROOM ? FM / 2 : FM / 4;
  constexpr int RW = WR * 32 * FMP;                // rows of a part
  constexpr int PR = CW / VO, NPC = RW * PR / NT;  // pieces of a row, pieces a lane stores
  constexpr int MP = FM / FMP, PARTS = FN / FNP * MP;
  static_assert(FMP >= 1 && RW * CW * TOB <= ROOM && NPC * NT == RW * PR, "whole parts that fit");
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, h = lane >> 5;
  const int wrow = wave / WC, wcol = wave % WC;
  TO* const y = static_cast<TO*>(a.y);
  // where a part's piece i of this lane belongs, and the elements left of its row
  auto place = [&](int part, int i, int64_t* at) {
    const int p = threadIdx.x + NT * i, lr = p / PR;
    const int r = lr / (32 * FMP) * (BM / WR) + 32 * (part % MP * FMP) + lr % (32 * FMP);
    const int col = n0 + WC * 32 * (part / MP * FNP) + p % PR * VO;
    *at = (j.begin + r) * a.cols + col;
    return r < j.nrow ? a.cols - col : 0;
  };
  u32x4_t g[2][NPC];
  auto ask = [&](int part) {
#pragma unroll
    for (int i = 0; i < NPC; ++i) {
      int64_t at;
      const int left = place(part, i, &at);
      g[part & 1][i] = load_left<TO, WHOLE>(static_cast<const TO*>(a.mask) + at, left);
    }
  };
  if constexpr (MASK && WHOLE) ask(0);
#pragma unroll
  for (int part = 0; part < PARTS; ++part) {
    if constexpr (MASK && WHOLE) {
      if (part + 1 < PARTS) ask(part + 1);
    }
    __syncthreads();
#pragma unroll
    for (int f = 0; f < FNP; ++f)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        // 4 adjacent columns of one row in every four registers of a lane
        const int c = col_of<WC>(wcol, f) + 8 * q + 4 * h, np = part / MP * FNP;
        const float4 b = *reinterpret_cast<const float4*>(s_bias + WC * 32 * np + c);
        const float bias[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
        for (int m = 0; m < FMP; ++m) {
          const int r = wrow * 32 * FMP + 32 * m + (lane & 31);
          float v[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            v[i] = acc[np + f][part % MP * FMP + m][4 * q + i] + bias[i];
            if (RELU) v[i] = v[i] < 0.0f ? 0.0f : v[i];
          }
          put4(reinterpret_cast<TO*>(lds + out_at<TO, CW>(r, c / VO)) + c % VO, v);
        }
      }
    if constexpr (MASK && !WHOLE) ask(part);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NPC; ++i) {
      int64_t at;
      const int left = place(part, i, &at), p = threadIdx.x + NT * i;
      if (left <= 0) continue;
      u32x4_t u = lds[out_at<TO, CW>(p / PR, p % PR)];
      if constexpr (MASK) {
        float v[VO], z[VO];
        unpack(u, v);
        unpack(g[part & 1][i], z);
#pragma unroll
        for (int e = 0; e < VO; ++e) v[e] = z[e] <= 0.0f ? 0.0f : v[e];
        u = pack(v);
      }
      store_left<TO, (BM * BN > 128 * 128)>(y + at, u, left);
    }
  }
}
// Small fp32 tiles leave from the registers, 32 bytes of a row by two lanes: without
// room for them in LDS a compute unit holds four workgroups rather than three (fp32 512
// -> 512, 8,000 positions: 53 us against 57; bf16 256 -> 64 to fp32, 348,208: 50 against
// 54).
template <bool MASK, bool WHOLE, bool RELU, int FM, int FN, int WR, int WC>
__device__ __forceinline__ void store_tile_direct(const f32x16 (&acc)[FN][FM], const float* s_bias,
                                                  const GroupedArgs& a, const Job& j, int n0) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, h = lane >> 5;
  float* const y = static_cast<float*>(a.y);
#pragma unroll
  for (int m = 0; m < FM; ++m) {
    const int r = wave / WC * FM * 32 + 32 * m + (lane & 31);
    const int64_t row = (j.begin + r) * a.cols + n0;
#pragma unroll
    for (int n = 0; n < FN; ++n) {
      const int c0 = col_of<WC>(wave % WC, n) + 4 * h;
      u32x4_t g[4];
      if constexpr (MASK) {
#pragma unroll
        for (int q = 0; q < 4; ++q)
          g[q] = load_left<float, WHOLE>(static_cast<const float*>(a.mask) + row + c0 + 8 * q,
                                         r < j.nrow ? a.cols - n0 - c0 - 8 * q : 0);
      }
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int c = c0 + 8 * q, left = r < j.nrow ? a.cols - n0 - c : 0;
        if (left <= 0) continue;
        const float4 b = *reinterpret_cast<const float4*>(s_bias + c);
        const float bias[4] = {b.x, b.y, b.z, b.w};
        float v[4], z[4];
        if constexpr (MASK) unpack(g[q], z);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          v[i] = acc[n][m][4 * q + i] + bias[i];
          if (RELU) v[i] = v[i] < 0.0f ? 0.0f : v[i];
          if (MASK) v[i] = z[i] <= 0.0f ? 0.0f : v[i];
        }
        store_left(y + row + c, pack(v), left);
      }
    }
  }
}
// The forward (BT false) has a ReLU and no mask, the input gradient a mask.
template <typename TO, bool BT, bool DIRECT, int BM, int BN, int WR, int WC, int BYTES>
__device__ __forceinline__ void store_tile(
    u32x4_t* lds, const f32x16 (&acc)[BN / WC / 32][BM / WR / 32], const float* s_bias,
    const GroupedArgs& a, const Job& j, int n0) {
  auto store = [&](auto mask, auto whole, auto relu) {
    if constexpr (DIRECT)
      store_tile_direct<mask.value, whole.value, relu.value, BM / WR / 32, BN / WC / 32, WR, WC>(
          acc, s_bias, a, j, n0);
    else
      store_tile_rows<TO, mask.value, whole.value, relu.value, BM, BN, WR, WC, BYTES>(
          lds, acc, s_bias, a, j, n0);
  };
  constexpr std::true_type yes;
  constexpr std::false_type no;
  constexpr std::bool_constant<BT> masks;
  constexpr std::bool_constant<!BT> relus;
  if (BT && a.mask && a.cols % Row<TO>::VEC == 0) store(masks, yes, no);
  else if (BT && a.mask) store(masks, no, no);
  else if (!BT && a.relu) store(no, yes, relus);
  else store(no, yes, no);
}

// Rows x weights: BT false: w[e] is [red][cols] (the forward), BT true: w[e] is
// [cols][red] (the input gradient).  A workgroup of WR x WC waves takes a tile of
// BM positions by BN columns, in stages of 64 bytes of the reduction through a
// ring of three or four LDS buffers: two or three stages are on their way while one is
// multiplied, one barrier a stage.  Sums stay in fp32 and are rounded once, after bias and ReLU
// or mask.  Whole 16-byte pieces at aligned addresses only (k_grouped_any takes the
// others).  Neither matrix cores nor LDS are its bound: of the cycles a compute unit has
// work, the matrix cores are busy in 34 % and the LDS in 17 (256 x 256 bf16, reductions
// of 1024), or in 56 to 60 % and 9 to 15 (64 x 64 fp32, reductions of 96 and 200); in the
// others the waves wait, for the stages of a tile that begins, at barriers, for stores.
// 65,536 x 2048 -> 2048 bf16: 603 us, 912 TFLOP/s (a large library product 1,175);
// 696,416 x 1024 -> 256 with a mask, backwards: 581 us, 628; 65,536 x 1024 -> 1024
// fp32: 1,160 us, 118 TFLOP/s (154).
template <typename T, typename TO, bool BT, int BM, int BN, int WR, int WC, int kRing>
__global__ __launch_bounds__(64 * WR * WC, 2) void k_grouped(GroupedArgs a) {
  constexpr int KB = 64;
  typedef RTile<T, BM, KB> TA;
  typedef RTile<T, BN, KB> TBr;
  typedef KTile<T, BN, KB> TBk;
  constexpr int VEC = Row<T>::VEC, BK = kBK<T, KB>, NT = 64 * WR * WC;
  constexpr int FM = BM / WR / 32, FN = BN / WC / 32;
  constexpr int PA = TA::PIECES / NT, PB = TBk::PIECES / NT;   // (as many as TBr's)
  constexpr int NP = TA::PIECES + TBk::PIECES;
  static_assert(NT % 256 == 0, "a lane's pieces of a stage have one place in their rows");
  // (the first one also takes the finished tile; separate arrays, so that the
  // compiler knows which loads a read waits for)
  constexpr int kOut = BM * BN * static_cast<int>(sizeof(TO)) / 16;
  constexpr bool kDirect = sizeof(TO) == 4 && BM == 64;
  constexpr int NP0 = kOut > NP && BM == 64 && !kDirect ? kOut : NP;
  __shared__ u32x4_t s_buf0[NP0], s_buf1[NP], s_buf2[NP], s_buf3[kRing == 4 ? NP : 1];
  __shared__ __attribute__((aligned(16))) float s_bias[BN];
  const T* const x = static_cast<const T*>(a.x);
  Job j;
  if (!grouped_job<TO, BM>(a, BN, &j)) return;
  const T* const w = static_cast<const T*>(a.w) + static_cast<int64_t>(j.group) * a.red * a.cols;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  load_bias<BN>(a, j, j.n0, s_bias);

  // What this lane stages of the rows: rows ra0 + NT / PR * i, of each the piece
  // that belongs at its place in LDS.  A row that is not there is read as zeros,
  // at one place all along (step 0).
  constexpr int PR = TA::PR;
  const T* const zero = reinterpret_cast<const T*>(&g_zeros);
  const int ra0 = threadIdx.x / PR, ka = (TA::at(ra0, threadIdx.x % PR) - ra0 * PR) * VEC;
  const T* pa[PA];
  int step[PA];
#pragma unroll
  for (int i = 0; i < PA; ++i) {
    const int64_t src = source_row(a, j, ra0 + NT / PR * i);
    step[i] = src >= 0 ? BK : 0;
    pa[i] = src >= 0 ? x + src * a.red + ka : zero;
  }
  const int nk = (a.red + BK - 1) / BK;
  // And of the weights, from the stage's own place; columns past the last one
  // are read as others (nothing of them is stored).
  const int kb = threadIdx.x / TBk::PR;            // (BT false) first row of the stage
  uint32_t pb[PB];
#pragma unroll
  for (int i = 0; i < PB; ++i) {
    if constexpr (BT) {
      const int n = ra0 + NT / PR * i;
      pb[i] = static_cast<uint32_t>(j.n0 + n < a.cols ? n : 0) * a.red + ka;
    } else {
      const int n = (TBk::at(kb, threadIdx.x % TBk::PR) - kb * TBk::PR) * VEC;
      pb[i] = static_cast<uint32_t>(kb + NT / TBk::PR * i) * a.cols + (j.n0 + n < a.cols ? n : 0);
    }
  }
  // Stages past the last one are asked for too, as zeros, so that the number of
  // loads behind a stage's own is known.
  int rk = 0;                                      // the next stage to request
  auto request = [&](u32x4_t* buf) {
    const int left = a.red - rk;                   // of the reduction
    const T* const ws = BT ? w + static_cast<int64_t>(j.n0) * a.red + rk
                           : w + static_cast<int64_t>(rk) * a.cols + j.n0;
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
        load_to_lds((BT ? ka : kb + NT / TBk::PR * i) < left ? ws + pb[i] : zero,
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
        acc, [&](int m, int q) { return rows_of(buf, m, q); },
        [&](int n, int q) { return weights_of(buf + TA::PIECES, BT ? WC * n : n, q); });
  };
  request(s_buf0);
  request(s_buf1);
  if constexpr (kRing == 4) {
    request(s_buf2);
    for (int s = 0; s < nk; s += kRing) {
      stage(s_buf0, s_buf3);
      if (s + 1 < nk) stage(s_buf1, s_buf0);
      if (s + 2 < nk) stage(s_buf2, s_buf1);
      if (s + 3 < nk) stage(s_buf3, s_buf2);
    }
  } else {
    for (int s = 0; s < nk; s += kRing) {
      stage(s_buf0, s_buf2);
      if (s + 1 < nk) stage(s_buf1, s_buf0);
      if (s + 2 < nk) stage(s_buf2, s_buf1);
    }
  }
  stage_barrier<0>();                              // (no load is on its way to s_buf0)
  store_tile<TO, BT, kDirect, BM, BN, WR, WC, NP0 * 16>(s_buf0, acc, s_bias, a, j, j.n0);
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

// A wave's finished FM x 2 blocks, rows r0 .. of the job, columns c0 .. c0 + 63 (of
// whole pieces), straight from the registers.  The halves of the wave exchange so
// that a lane has all 32 columns of one block of its row, and the lanes of a quad
// so that four of them store 64 adjacent bytes of one row at a time.
template <typename TO, int FM, bool RELU, bool MASK>
__device__ __forceinline__ void store_wave_rows(const f32x16 (&acc)[2][FM], const GroupedArgs& a,
                                                const Job& j, int r0, int c0) {
  constexpr int VO = Row<TO>::VEC, TOB = static_cast<int>(sizeof(TO));
  constexpr int NU = 8 * TOB, W4 = TOB;            // words of 32 columns, of 4
  const int lane = threadIdx.x & 63, h = lane >> 5;
  const int64_t base = (j.begin + r0 + (lane & 28)) * a.cols;
#pragma unroll
  for (int m = 0; m < FM; ++m) {
    // u[n]: this lane's words of block n, those of 4 columns of every 8
    uint32_t u[2][NU / 2];
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        float v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          v[i] = acc[n][m][4 * q + i];
          if (RELU) v[i] = v[i] < 0.0f ? 0.0f : v[i];
        }
        if constexpr (TOB == 2) {
          u[n][2 * q] = pack2(v[0], v[1]);
          u[n][2 * q + 1] = pack2(v[2], v[3]);
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) u[n][4 * q + i] = __float_as_uint(v[i]);
        }
      }
    // word[k]: the row's words of block h in order
    uint32_t word[NU];
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
      for (int i = 0; i < W4; ++i) {
        const auto r = __builtin_amdgcn_permlane32_swap(u[0][W4 * q + i], u[1][W4 * q + i], false,
                                                        false);
        word[2 * W4 * q + i] = r[0];
        word[2 * W4 * q + W4 + i] = r[1];
      }
#pragma unroll
    for (int half = 0; half < NU / 16; ++half) {
      // 64 bytes of each of the quad's rows: piece p of lane i is words 4 p .. + 3
      u32x4_t piece[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t v[4];
#pragma unroll
        for (int p = 0; p < 4; ++p) v[p] = word[16 * half + 4 * p + i];
        quad_transpose(v);
#pragma unroll
        for (int p = 0; p < 4; ++p) piece[p][i] = v[p];
      }
      // now piece[t] is piece lane % 4 of the row of the quad's lane t
      const int col = c0 + 32 * h + (16 * half + 4 * (lane & 3)) * 4 / TOB;
      const int rows = col < a.cols ? j.nrow - r0 - 32 * m - (lane & 28) : 0;
      const int64_t at = base + static_cast<int64_t>(32 * m) * a.cols + col;
      TO* const y = static_cast<TO*>(a.y) + at;
      u32x4_t g[4];
      if constexpr (MASK) {
        const TO* const mask = static_cast<const TO*>(a.mask) + at;
#pragma unroll
        for (int t = 0; t < 4; ++t)
          g[t] = load_left<TO, true>(mask + static_cast<int64_t>(t) * a.cols, t < rows ? VO : 0);
      }
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        if constexpr (MASK) {
          float v[VO], z[VO];
          unpack(piece[t], v);
          unpack(g[t], z);
#pragma unroll
          for (int e = 0; e < VO; ++e) v[e] = z[e] <= 0.0f ? 0.0f : v[e];
          piece[t] = pack(v);
        }
        if (t < rows) store_piece_past(y + static_cast<int64_t>(t) * a.cols, piece[t]);
      }
    }
  }
}

// Short reductions of bf16 (NK stages of 32): a workgroup keeps its 256 rows in
// registers, as fragments, and takes the columns `span` by 128 at a time.  Only
// the weights go through LDS, a ring of 6 or 8 stages of them, all but one on their
// way while that one is multiplied, and finished tiles leave from the registers.
// (k_grouped would read the rows once per 256 columns, and drain and refill for
// every tile of a few stages.)  The ring is as long as that because a wave's loads
// and stores are counted together and in order: with 4 stages of 64 ahead a stage
// waited for the stores of the tile before, 669 us instead of 591 for 256 -> 1024
// at 696,416 positions, and two workgroups of 128 rows a compute unit took 621.
// (570 to 630 us from card to card, 580 to 640 TFLOP/s: the 1.4 GB of outputs alone
// would take 210 at the fastest stores, and wait for the products of their tile.)
constexpr int short_ring(int nk) { return nk == 6 ? 6 : 8; }
template <typename TO, bool BT, int NK, bool RELU, bool MASK>
__global__ __launch_bounds__(512, 2) void k_grouped_short(GroupedArgs a, int span) {
  typedef bf16_t T;
  typedef Mma<T> M;
  constexpr int BM = kShortRows, BN = 128, NT = 512, WC = 2, FM = 2, FN = 2;
  constexpr int kRing = short_ring(NK), U = kRing / NK;   // tiles until the ring repeats
  constexpr int KB = 64;
  typedef RTile<T, BN, KB> TBr;
  typedef KTile<T, BN, KB> TBk;
  constexpr int VEC = Row<T>::VEC, BK = kBK<T, KB>, STEPS = BK / M::KS;
  constexpr int PB = TBk::PIECES / NT;
  // (separate arrays, so that the compiler knows which loads a read waits for)
  constexpr int NP = TBk::PIECES;
  __shared__ u32x4_t s_w0[NP], s_w1[NP], s_w2[NP], s_w3[NP], s_w4[NP], s_w5[NP],
      s_w6[kRing > 6 ? NP : 1], s_w7[kRing > 6 ? NP : 1];
  const T* const x = static_cast<const T*>(a.x);
  Job j;
  if (!grouped_job<TO, BM>(a, span, &j)) return;
  const T* const w = static_cast<const T*>(a.w) + static_cast<int64_t>(j.group) * a.red * a.cols;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int wr = wave / WC * 64, wc = wave % WC * 64;
  const T* const zero = reinterpret_cast<const T*>(&g_zeros);
  const int end = a.cols - j.n0 < span ? a.cols : j.n0 + span;
  // A lane's pieces of a weights' stage are those that belong at its place in LDS.
  // Stages past the last one are asked for too (as zeros or as columns of others),
  // so that the number of loads behind a stage's own is known.
  constexpr int PR = TBr::PR;
  const int ra0 = threadIdx.x / PR, ka = (TBr::at(ra0, threadIdx.x % PR) - ra0 * PR) * VEC;
  const int kb = threadIdx.x / TBk::PR;
  const int nb = (TBk::at(kb, threadIdx.x % TBk::PR) - kb * TBk::PR) * VEC;
  // (columns past the last one are read as others: nothing of them is stored)
  const int own = lane_place(BT ? ra0 * a.red + ka : kb * a.cols + nb);
  const int next = BT ? NT / PR * a.red : NT / TBk::PR * a.cols;
  auto request = [&](int k, int n0, u32x4_t* buf) {
    const bool whole = n0 + BN <= a.cols && (k + 1) * BK <= a.red;
    const T* const ws = w + (BT ? static_cast<int64_t>(n0) * a.red + k * BK
                                : static_cast<int64_t>(k) * BK * a.cols + n0);
    if (whole) {
#pragma unroll
      for (int i = 0; i < PB; ++i) load_to_lds(ws + (own + i * next), buf + NT * i + 64 * wave);
    } else {
#pragma unroll
      for (int i = 0; i < PB; ++i) {
        const int n = n0 + (BT ? ra0 + NT / PR * i : nb);
        const int c = k * BK + (BT ? ka : kb + NT / TBk::PR * i);
        load_to_lds(n < a.cols && c < a.red ? ws + (own + i * next) : zero,
                    buf + NT * i + 64 * wave);
      }
    }
  };
  const std::conditional_t<BT, typename TBr::Reader, typename TBk::template Reader<32, FN>>
      weights_of(wc, lane);
  auto ring = [&](int r) {
    return r < 4 ? (r < 2 ? (r ? s_w1 : s_w0) : (r > 2 ? s_w3 : s_w2))
                 : (r < 6 ? (r > 4 ? s_w5 : s_w4) : (r > 6 ? s_w7 : s_w6));
  };
  // A tile starts from its bias: lane i has that of column wc + i, asked for a
  // tile before.
  const float* const b = a.bias ? a.bias + static_cast<int64_t>(j.group) * a.cols : nullptr;
  auto bias_of = [&](int n0) {
    const int c = n0 + wc + lane;
    return b && c < a.cols ? b[c] : 0.0f;
  };
  // The rows.
  typename M::Frag fa[FM][NK * STEPS];
#pragma unroll
  for (int m = 0; m < FM; ++m) {
    const int64_t src = source_row(a, j, wr + 32 * m + (lane & 31));
    const T* const p = x + (src < 0 ? 0 : src) * a.red;
#pragma unroll
    for (int q = 0; q < NK * STEPS; ++q) {
      const int c = 16 * q + 8 * (lane >> 5);
      fa[m][q] = __builtin_bit_cast(typename M::Frag,
                                    load_left<T, true>(p + c, src < 0 ? 0 : a.red - c));
    }
  }
  float bias = bias_of(j.n0);
#pragma unroll
  for (int s = 0; s < kRing - 1; ++s) request(s % NK, j.n0 + s / NK * BN, ring(s));
  for (int n1 = j.n0; n1 < end; n1 += U * BN) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int n0 = n1 + u * BN;
      if (n0 >= end) break;
      f32x16 acc[FN][FM];
#pragma unroll
      for (int n = 0; n < FN; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float v = __shfl(bias, 32 * n + 8 * (i / 4) + 4 * (lane >> 5) + i % 4, 64);
#pragma unroll
          for (int m = 0; m < FM; ++m) acc[n][m][i] = v;
        }
      bias = bias_of(n0 + BN);
#pragma unroll
      for (int k = 0; k < NK; ++k) {
        const int s = u * NK + k;                  // (of the ring's U tiles)
        u32x4_t* const buf = ring(s);
        // kRing - 2 stages' loads are behind this one's
        stage_barrier<PB * (kRing - 2)>();
        const int ahead = s + kRing - 1;
        request(ahead % NK, n1 + ahead / NK * BN, ring(ahead % kRing));
#pragma unroll
        for (int q = 0; q < STEPS; ++q) {
          typename M::Frag fb[FN];
#pragma unroll
          for (int n = 0; n < FN; ++n) fb[n] = weights_of(buf, n, q);
#pragma unroll
          for (int n = 0; n < FN; ++n)
#pragma unroll
            for (int m = 0; m < FM; ++m)
              acc[n][m] = M::mma(fb[n], fa[m][k * STEPS + q], acc[n][m]);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      store_wave_rows<TO, FM, RELU, MASK>(acc, a, j, wr, n0 + wc);
    }
  }
  stage_barrier<0>();                              // (no load to LDS outlives the workgroup)
}

// The same for rows and weights whose pieces may be cut (widths that are no
// multiple of a piece) or unaligned: through registers, 128 x 128 or 64 x 64 by
// four waves in 2 x 2.  (100,000 x 500 -> 250 backwards: 57 us bf16, 439 TFLOP/s, 277
// fp32, 90.)
template <typename T, typename TO, bool BT, int BM, int BN>
__global__ __launch_bounds__(kThreads, 2) void k_grouped_any(GroupedArgs a) {
  constexpr int KB = 128;
  typedef RTile<T, BM, KB> TA;
  typedef RTile<T, BN, KB> TBr;
  typedef KTile<T, BN, KB> TBk;
  constexpr int VEC = Row<T>::VEC, BK = kBK<T, KB>;
  constexpr int FM = BM / 64, FN = BN / 64;
  constexpr int PA = TA::PIECES / kThreads, PB = TBk::PIECES / kThreads;
  constexpr int NP = TA::PIECES + TBk::PIECES;
  __shared__ u32x4_t s_buf[NP];
  __shared__ __attribute__((aligned(16))) float s_bias[BN];
  const T* const x = static_cast<const T*>(a.x);
  Job j;
  if (!grouped_job<TO, BM>(a, BN, &j)) return;
  const int n0 = j.n0;
  load_bias<BN>(a, j, n0, s_bias);
  const T* const w = static_cast<const T*>(a.w) + static_cast<int64_t>(j.group) * a.red * a.cols;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int ra0 = threadIdx.x >> 3, ka = (threadIdx.x & 7) * VEC;
  const T* pa[PA];
  bool oka[PA];
#pragma unroll
  for (int i = 0; i < PA; ++i) {
    const int64_t src = source_row(a, j, ra0 + 32 * i);
    oka[i] = src >= 0;
    pa[i] = x + (src < 0 ? 0 : src) * a.red;
  }
  u32x4_t ra[PA], rb[PB];
  auto request = [&](int k0, int n0) {
#pragma unroll
    for (int i = 0; i < PA; ++i)
      ra[i] = load_left<T, false>(pa[i] + k0 + ka, oka[i] ? a.red - k0 - ka : 0);
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
  request(0, n0);
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
    if (k0 + BK < a.red) request(k0 + BK, n0);
    multiply_stage<T, KB, FM, FN>(
        acc, [&](int m, int q) { return rows_of(s_buf, m, q); },
        [&](int n, int q) { return weights_of(s_buf + TA::PIECES, BT ? 2 * n : n, q); });
  }
  store_tile<TO, BT, false, BM, BN, 2, 2, NP * 16>(s_buf, acc, s_bias, a, j, n0);
}

// Few positions in all (a row at a time through its experts): the weights' bytes,
// once, and the time to the last of them are all there is.  A workgroup of 16 waves
// takes up to 4 positions of a group and 64 bytes of columns, 4 lanes side by side;
// its 256 slices of the reduction run down the weights' rows on the vector ALU, 8
// loads of a slice in flight, and are added over the lanes, then the waves, in
// order.  (The tiles' chain of stages took 48 us for one fp32 position of 2048 ->
// 512, this 7.8.)
constexpr int kFewThreads = 1024;
// v of lane i + D within 16 lanes (rotating), D = 4 or 8
template <int D> __device__ __forceinline__ float row_rotate(float v) {
  return __uint_as_float(static_cast<uint32_t>(__builtin_amdgcn_update_dpp(
      0, static_cast<int>(__float_as_uint(v)), 0x120 | D, 0xf, 0xf, true)));
}
template <typename T, typename TO>
__global__ __launch_bounds__(kFewThreads) void k_grouped_few(GroupedArgs a) {
  constexpr int VEC = Row<T>::VEC, R = 4, CL = 4, NC = CL * VEC, KS = kFewThreads / CL;
  constexpr int KC = 2048, UN = 8;                 // of the reduction in LDS; loads in flight
  constexpr int NW = kFewThreads / 64;
  __shared__ float s_x[R][KC];
  __shared__ float s_sum[NW][R][NC];
  const T* const x = static_cast<const T*>(a.x);
  Job j;
  if (!grouped_job<TO, R>(a, NC, &j)) return;
  const T* const w = static_cast<const T*>(a.w) + static_cast<int64_t>(j.group) * a.red * a.cols;
  const int slice = threadIdx.x / CL, c = j.n0 + threadIdx.x % CL * VEC;
  float acc[R][VEC];
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int i = 0; i < VEC; ++i) acc[r][i] = 0.0f;
  const int sr = threadIdx.x / (kFewThreads / R);  // the row a lane stages
  const int64_t src = source_row(a, j, sr);
  for (int k0 = 0; k0 < a.red; k0 += KC) {
    const int kc = a.red - k0 < KC ? a.red - k0 : KC;
    __syncthreads();
    for (int k = threadIdx.x % (kFewThreads / R); k < kc; k += kFewThreads / R)
      s_x[sr][k] = src >= 0 ? Row<T>::get(x[src * a.red + k0 + k]) : 0.0f;
    __syncthreads();
    for (int k1 = slice; k1 < kc; k1 += KS * UN) {
      u32x4_t u[UN];
#pragma unroll
      for (int i = 0; i < UN; ++i) {
        const int k = k1 + KS * i;
        u[i] = load_piece(k < kc && c < a.cols ? w + static_cast<int64_t>(k0 + k) * a.cols + c
                                               : reinterpret_cast<const T*>(&g_zeros));
      }
#pragma unroll
      for (int i = 0; i < UN; ++i) {
        const int k = k1 + KS * i;
        if (k >= kc) break;
        float v[VEC];
        unpack(u[i], v);
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
          for (int e = 0; e < VEC; ++e) acc[r][e] = fmaf(s_x[r][k], v[e], acc[r][e]);
      }
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
  TO* const y = static_cast<TO*>(a.y);
  if (threadIdx.x < R * NC) {
    const int r = threadIdx.x / NC, col = j.n0 + threadIdx.x % NC;
    if (r >= j.nrow || col >= a.cols) return;
    float z = 0.0f;
#pragma unroll
    for (int q = 0; q < NW; ++q) z += s_sum[q][r][threadIdx.x % NC];
    if (a.bias) z += a.bias[static_cast<int64_t>(j.group) * a.cols + col];
    if (a.relu && z < 0.0f) z = 0.0f;
    y[(j.begin + r) * a.cols + col] = Row<TO>::put(z);
  }
}

// Weight gradient of a BC x BN tile of one group, over a chunk of its
// positions: dw[c][n] = sum_j x[row j][c] dy[j][n].  Both operands are staged
// with the positions as the reduction's rows.  Chunk `job` leaves its sums as
// part[job] (one chunk per group: dw[group] itself).  The workgroups of the
// first rows of dw also sum dy.  No atomics: the chunks are added in their order.
// Bound as k_grouped (matrix cores 29 % of the busy cycles, LDS 12; fp32 60 and 8), and
// by the gathered rows' latency: 696,416 positions of 16 x 256 x 1024 bf16 take 680 us and
// 50 for the chunks' sums, 500 TFLOP/s in all; 59,520 of 8 x 96 x 200 fp32 52 + 9 us (38
// TFLOP/s, three quarters of each tile filled).
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

// DMA: whole 16-byte pieces at aligned addresses, straight to LDS, through a ring of
// four buffers as k_grouped's, of three for tiles below 256, so that one workgroup
// more fits a compute unit (fp32 512 x 512 of 8 groups, 65,536 positions: 450 -> 408
// us); else through registers, one buffer.
template <typename T, int BC, int BN, int WR, int WC, bool DMA>
__global__ __launch_bounds__(64 * WR * WC, 2) void k_grouped_dw(WeightArgs a) {
  constexpr int KB = DMA ? 64 : 128, kRing = BC == 256 ? 4 : 3;
  typedef KTile<T, BC, KB> TX;
  typedef KTile<T, BN, KB> TY;
  constexpr int VEC = Row<T>::VEC, BK = kBK<T, KB>, NT = 64 * WR * WC;
  constexpr int FC = BC / WR / 32, FN = BN / WC / 32;
  constexpr int PX = TX::PIECES / NT, PY = TY::PIECES / NT, NP = TX::PIECES + TY::PIECES;
  static_assert(NT % 256 == 0, "a lane's pieces of a stage have one place in their rows");
  constexpr int NR = DMA ? NP : 1;
  __shared__ u32x4_t s_buf0[NP], s_buf1[NR], s_buf2[NR], s_buf3[kRing == 4 ? NR : 1];
  // The row numbers of NT positions at a time, three such runs: the one being
  // requested, the next one, and the one a slower wave may still read.
  __shared__ int32_t s_row[3][NT];
  const T *const x = static_cast<const T*>(a.x), *const dy = static_cast<const T*>(a.dy);
  const int64_t nc = (a.C_in + BC - 1) / BC, nn = (a.C_out + BN - 1) / BN;
  const int64_t id = die_order(blockIdx.x, gridDim.x);
  const int64_t job = id / (nc * nn);
  const int c0 = static_cast<int>(id / nn % nc) * BC, n0 = static_cast<int>(id % nn) * BN;
  Tile t;
  if (a.chunk) {
    t = find_tile<false>(a.offsets, a.E, a.m, a.chunk, job);
    if (t.group < 0) return;
  } else {
    const int32_t begin = clamp_offset(a.offsets[job], a.m);
    const int32_t end = clamp_offset(a.offsets[job + 1], a.m);
    t = Tile{static_cast<int>(job), begin, end < begin ? begin : end, 0};
  }
  constexpr int RUN = NT / BK;                     // stages of a run
  auto row_of = [&](int64_t j) {
    return j >= t.end ? -1 : a.rows ? a.rows[j] : static_cast<int32_t>(j);
  };
  int64_t rj = t.begin;                            // the next stage to request
  int rq = 0, run = 0;                             // its place in its run, its run (mod 3)
  int32_t row_next = 0;
  auto first_rows = [&] {
    s_row[0][threadIdx.x] = row_of(rj + threadIdx.x);
    row_next = row_of(rj + NT + threadIdx.x);
  };
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  first_rows();
  if (!a.chunk && t.end > t.begin) {               // (uniform, as below)
    // The group's own offset is meant to be the largest up to it: found out while the
    // row numbers come, and mended where it is not (group_span).
    const auto larger = [](uint32_t u, uint32_t v) { return u > v ? u : v; };
    uint32_t top = wave_reduce(part_top<NT>(a.offsets, a.m, t.group), larger);
    __shared__ uint32_t s_top[NT / 64];
    if (lane == 0) s_top[wave] = top;
    __syncthreads();
#pragma unroll
    for (int q = 0; q < NT / 64; ++q) top = larger(top, s_top[q]);
    top = __builtin_amdgcn_readfirstlane(top);     // (known to the compiler as uniform)
    if (top > t.begin) {
      rj = t.begin = top;
      if (t.end < t.begin) t.end = t.begin;
      first_rows();
      __syncthreads();
    }
  } else {
    __syncthreads();
  }
  // a lane's first row of a stage and its column there, per operand: the place
  // in LDS that a lane's piece goes to is its own (DMA) or its piece's
  const int jx = threadIdx.x / TX::PR, px = threadIdx.x % TX::PR;
  const int jy = threadIdx.x / TY::PR, py = threadIdx.x % TY::PR;
  const int cx = c0 + (DMA ? TX::at(jx, px) - jx * TX::PR : px) * VEC;
  const int cy = n0 + (DMA ? TY::at(jy, py) - jy * TY::PR : py) * VEC;
  // (DMA) columns past the last one are read as others: nothing of them is stored
  const int cxr = cx < a.C_in ? cx : 0, cyr = cy < a.C_out ? cy : 0;
  u32x4_t rx[DMA ? 1 : PX], ry[DMA ? 1 : PY];
  auto request = [&](u32x4_t* buf) {
    const T* const zero = reinterpret_cast<const T*>(&g_zeros);
#pragma unroll
    for (int i = 0; i < PX; ++i) {
      const int32_t row = s_row[run][rq * BK + jx + NT / TX::PR * i];
      const bool ok = row >= 0 && row < a.n_x;
      const T* const p = x + static_cast<int64_t>(row) * a.C_in;
      if constexpr (DMA) load_to_lds(ok ? p + cxr : zero, buf + NT * i + 64 * wave);
      else rx[i] = load_left<T, false>(p + cx, ok ? a.C_in - cx : 0);
    }
#pragma unroll
    for (int i = 0; i < PY; ++i) {
      const int64_t j = rj + jy + NT / TY::PR * i;
      const T* const p = dy + j * a.C_out;
      if constexpr (DMA)
        load_to_lds(j < t.end ? p + cyr : zero, buf + TX::PIECES + NT * i + 64 * wave);
      else ry[i] = load_left<T, false>(p + cy, j < t.end ? a.C_out - cy : 0);
    }
    if (rq == 0) {
      // (read RUN - 1 stages on at the earliest, with barriers between)
      s_row[run == 2 ? 0 : run + 1][threadIdx.x] = row_next;
      row_next = row_of(rj + 2 * NT + threadIdx.x);
    }
    rj += BK;
    if (++rq == RUN) {
      rq = 0;
      run = run == 2 ? 0 : run + 1;
    }
  };
  const int wr = wave / WC * (BC / WR), wc = wave % WC * (BN / WC);
  const bool bias = a.db && c0 == 0 && wr == 0;    // (uniform over the wave)
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
  auto multiply = [&](const u32x4_t* buf) {
    multiply_stage<T, KB, FC, FN>(
        acc, [&](int m, int q) { return x_of(buf, m, q); },
        [&](int n, int q) {
          const typename Mma<T>::Frag f = dy_of(buf + TX::PIECES, n, q);
          if (bias) sum[n] = frag_sum(sum[n], f);
          return f;
        });
  };
  const int64_t nk = (t.end - t.begin + BK - 1) / BK;
  if constexpr (DMA) {
    // (stages past the last one are asked for too, as zeros)
    auto stage = [&](const u32x4_t* buf, u32x4_t* before) {
      stage_barrier<(PX + PY) * (kRing - 2)>();
      request(before);
      multiply(buf);
    };
    request(s_buf0);
    request(s_buf1);
    if constexpr (kRing == 4) {
      request(s_buf2);
      for (int64_t s = 0; s < nk; s += kRing) {
        stage(s_buf0, s_buf3);
        if (s + 1 < nk) stage(s_buf1, s_buf0);
        if (s + 2 < nk) stage(s_buf2, s_buf1);
        if (s + 3 < nk) stage(s_buf3, s_buf2);
      }
    } else {
      for (int64_t s = 0; s < nk; s += kRing) {
        stage(s_buf0, s_buf2);
        if (s + 1 < nk) stage(s_buf1, s_buf0);
        if (s + 2 < nk) stage(s_buf2, s_buf1);
      }
    }
    stage_barrier<0>();                            // (no load to LDS outlives the workgroup)
  } else {
    if (nk) request(nullptr);
    for (int64_t s = 0; s < nk; ++s) {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < PX; ++i) s_buf0[TX::at(jx + NT / TX::PR * i, px)] = rx[i];
#pragma unroll
      for (int i = 0; i < PY; ++i)
        s_buf0[TX::PIECES + TY::at(jy + NT / TY::PR * i, py)] = ry[i];
      __syncthreads();
      if (s + 1 < nk) request(nullptr);
      multiply(s_buf0);
    }
  }
  if (bias) {
#pragma unroll
    for (int n = 0; n < FN; ++n) {
      const float v = sum[n] + __shfl_xor(sum[n], 32, 64);
      const int col = n0 + wc + 32 * n + lane;
      if (lane < 32 && col < a.C_out) a.db[job * a.C_out + col] = v;
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

// The chunks' sums of a group: kThreads / RUNS lanes side by side with four values
// each, RUNS of them down the chunks, every RUNS-th one each, then those in order.
// The first workgroup of a group also adds up the bias gradient.  (Eight runs
// where few values have many chunks: 29 us of a gradient of 64 x 256 became 9.)
template <int RUNS>
__global__ __launch_bounds__(kThreads) void k_grouped_dw_sum(
    const float* __restrict__ part, const float* __restrict__ part_db,
    const int32_t* __restrict__ offsets, int E, int64_t m, int64_t chunk, int64_t per, int C_out,
    float* __restrict__ dw, float* __restrict__ db) {
  constexpr int kLanes = kThreads / RUNS;
  __shared__ f32x4_t s_sum[RUNS][kLanes];
  const int e = blockIdx.y, lane = threadIdx.x % kLanes, run = threadIdx.x / kLanes;
  // chunks before group e, and its own (every wave finds them)
  int64_t first = 0, count = 0;
  int32_t top = 0;
  for (int e0 = 0; e0 <= e; e0 += 64) {
    const Span s = group_span<false>(offsets, E, m, e0, &top);
    const int64_t c = (s.end - s.begin + chunk - 1) / chunk;
    const int g = e0 + static_cast<int>(threadIdx.x & 63);
    if (g < e) first += c; else if (g == e) count = c;
  }
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    first += __shfl_xor(first, d, 64);
    count += __shfl_xor(count, d, 64);
  }
  auto add = [&](const float* p, int64_t width, int64_t i, float* out) {
    f32x4_t a = {0.0f, 0.0f, 0.0f, 0.0f};
    if (i + 4 <= width) {
#pragma unroll 4
      for (int64_t c = run; c < count; c += RUNS)
        a += __builtin_bit_cast(f32x4_t, load_piece(p + (first + c) * width + i));
    } else {
      for (int64_t c = run; c < count; c += RUNS)
        for (int q = 0; q < 4 && i + q < width; ++q) a[q] += p[(first + c) * width + i + q];
    }
    if constexpr (RUNS > 1) {
      s_sum[run][lane] = a;
      __syncthreads();
    }
    if (run == 0 && i < width) {
#pragma unroll
      for (int q = 1; q < RUNS; ++q) a += s_sum[q][lane];
      store_left(out + e * width + i, __builtin_bit_cast(u32x4_t, a), width - i);
    }
    if constexpr (RUNS > 1) __syncthreads();
  };
  add(part, per, (static_cast<int64_t>(blockIdx.x) * kLanes + lane) * 4, dw);
  if (db && blockIdx.x == 0)
    for (int64_t c = 0; c < C_out; c += kLanes * 4) add(part_db, C_out, c + lane * 4, db);
}

// Whole aligned 16-byte pieces in rows of C elements from p.
template <typename T> bool whole_rows(const void* p, int64_t C) {
  return C % Row<T>::VEC == 0 && aligned_to(p, 16);
}

template <int BM>
bool grouped_grid(const GroupedArgs& a, int span, int threads, uint32_t* blocks) {
  const int64_t n = tile_bound(a.m, a.E + 1, BM) * ((a.cols + span - 1) / span);
  *blocks = static_cast<uint32_t>(n);
  return grid_fits(n, threads);
}
template <typename T, typename TO, bool BT, int BM, int BN, int WR, int WC, int RING = 4>
int run_grouped(const GroupedArgs& a) {
  uint32_t blocks;
  if (!grouped_grid<BM>(a, BN, 64 * WR * WC, &blocks)) return SPCONV_EINVAL;
  k_grouped<T, TO, BT, BM, BN, WR, WC, RING><<<blocks, 64 * WR * WC, 0, a.st>>>(a);
  return launched();
}
template <typename T, typename TO, bool BT, int BM, int BN>
int run_grouped_any(const GroupedArgs& a) {
  uint32_t blocks;
  if (!grouped_grid<BM>(a, BN, kThreads, &blocks)) return SPCONV_EINVAL;
  k_grouped_any<T, TO, BT, BM, BN><<<blocks, kThreads, 0, a.st>>>(a);
  return launched();
}
template <typename TO, bool BT, int NK> int run_grouped_short(const GroupedArgs& a) {
  // all columns, or as many as leave eight workgroups a compute unit
  const int64_t tiles = tile_bound(a.m, a.E + 1, kShortRows), want = 2048 / tiles + 1;
  const int ncol = (a.cols + 127) / 128;
  const int parts = static_cast<int>(want < ncol ? want : ncol);
  const int span = (ncol + parts - 1) / parts * 128;
  uint32_t blocks;
  if (!grouped_grid<kShortRows>(a, span, 512, &blocks)) return SPCONV_EINVAL;
  if (BT ? a.mask != nullptr : a.relu != 0)
    k_grouped_short<TO, BT, NK, !BT, BT><<<blocks, 512, 0, a.st>>>(a, span);
  else
    k_grouped_short<TO, BT, NK, false, false><<<blocks, 512, 0, a.st>>>(a, span);
  return launched();
}
// The kernel that grouped_plan says.
template <typename T, typename TO, bool BT> int by_size(const GroupedArgs& a) {
  const bool whole = whole_rows<T>(a.x, a.red) && whole_rows<T>(a.w, BT ? a.red : a.cols);
  const GroupedPlan p = grouped_plan(Row<T>::VEC == 4 ? SPCONV_F32 : SPCONV_BF16,
                                     Row<TO>::VEC == 4 ? SPCONV_F32 : SPCONV_BF16, BT, a.m, a.E,
                                     a.red, a.cols, whole);
  if constexpr (!BT) {
    if (p.kernel == GroupedKernel::kFew) {
      uint32_t blocks;
      if (!grouped_grid<4>(a, 4 * Row<T>::VEC, kFewThreads, &blocks)) return SPCONV_EINVAL;
      k_grouped_few<T, TO><<<blocks, kFewThreads, 0, a.st>>>(a);
      return launched();
    }
  }
  if (p.kernel == GroupedKernel::kAny)
    return p.tile == 64 ? run_grouped_any<T, TO, BT, 64, 64>(a)
                        : run_grouped_any<T, TO, BT, 128, 128>(a);
  if constexpr (sizeof(T) == 2) {
    if (p.kernel == GroupedKernel::kShort) {
      if (p.ring == 2) return run_grouped_short<TO, BT, 2>(a);
      if (p.ring == 4) return run_grouped_short<TO, BT, 4>(a);
      if (p.ring == 6) return run_grouped_short<TO, BT, 6>(a);
      return run_grouped_short<TO, BT, 8>(a);
    }
    if (p.tile == 256) return run_grouped<T, TO, BT, 256, 256, 2, 4>(a);
  }
  if (p.tile == 128) return run_grouped<T, TO, BT, 128, 128, 2, 2>(a);
  if (p.ring == 3) return run_grouped<T, TO, BT, 64, 64, 2, 2, 3>(a);
  return run_grouped<T, TO, BT, 64, 64, 2, 2>(a);
}
template <bool BT> int run_types(int in_dt, int out_dt, const GroupedArgs& a) {
  if (in_dt == SPCONV_BF16)
    return out_dt == SPCONV_BF16 ? by_size<bf16_t, bf16_t, BT>(a) : by_size<bf16_t, float, BT>(a);
  return out_dt == SPCONV_BF16 ? by_size<float, bf16_t, BT>(a) : by_size<float, float, BT>(a);
}

template <typename T> void run_dw(const WeightArgs& a, const DwPlan& p) {
  const uint32_t blocks = static_cast<uint32_t>(p.jobs * p.tiles);
  const bool dma = whole_rows<T>(a.x, a.C_in) && whole_rows<T>(a.dy, a.C_out);
  if constexpr (sizeof(T) == 2) {
    if (p.tile == 256) {
      k_grouped_dw<T, 256, 256, 2, 4, true><<<blocks, 512, 0, a.st>>>(a);
      return;
    }
  }
  if (p.tile == 128 && dma)
    k_grouped_dw<T, 128, 128, 2, 2, true><<<blocks, 256, 0, a.st>>>(a);
  else if (p.tile == 128)
    k_grouped_dw<T, 128, 128, 2, 2, false><<<blocks, 256, 0, a.st>>>(a);
  else if (dma)
    k_grouped_dw<T, 64, 64, 2, 2, true><<<blocks, 256, 0, a.st>>>(a);
  else
    k_grouped_dw<T, 64, 64, 2, 2, false><<<blocks, 256, 0, a.st>>>(a);
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
  // (the pointers are not known yet: enough for either kernel)
  const size_t a = dw_plan(dt, m, E, C_in, C_out, true).bytes;
  const size_t b = dw_plan(dt, m, E, C_in, C_out, false).bytes;
  *bytes = a > b ? a : b;
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
  const bool wide = dt == SPCONV_BF16
                        ? whole_rows<bf16_t>(x, C_in) && whole_rows<bf16_t>(dy, C_out)
                        : whole_rows<float>(x, C_in) && whole_rows<float>(dy, C_out);
  const DwPlan plan = dw_plan(dt, m, E, C_in, C_out, wide);
  if (!ptr_ok(x, n_x, e) || !ptr_ok(dy, m, e) || !ptr_ok(offsets, 1, 4) || !aligned_to(rows, 4) ||
      !ptr_ok(dw, 1, 4) || !aligned_to(db, 4) ||
      (plan.bytes && (!workspace || !aligned_to(workspace, 16) || workspace_bytes < plan.bytes)))
    return SPCONV_EINVAL;
  if (!grid_fits(plan.jobs * plan.tiles, 512)) return SPCONV_EINVAL;
  hipStream_t st = static_cast<hipStream_t>(stream);
  WeightArgs a{x, n_x, dy, offsets, rows, dw, db, m, plan.chunk, E, C_in, C_out, st};
  const int64_t per = static_cast<int64_t>(C_in) * C_out;
  if (plan.chunk) {
    a.dw = static_cast<float*>(workspace);
    a.db = db ? a.dw + plan.jobs * per : nullptr;
  }
  if (dt == SPCONV_BF16) run_dw<bf16_t>(a, plan); else run_dw<float>(a, plan);
  if (plan.chunk) {
    if (dw_sum_runs(plan, E, per) == 8) {
      const dim3 grid(static_cast<uint32_t>((per + kThreads / 2 - 1) / (kThreads / 2)), E);
      k_grouped_dw_sum<8><<<grid, kThreads, 0, st>>>(a.dw, a.db, offsets, E, m, plan.chunk, per,
                                                     C_out, dw, db);
    } else {
      const dim3 grid(static_cast<uint32_t>((per + 4 * kThreads - 1) / (4 * kThreads)), E);
      k_grouped_dw_sum<1><<<grid, kThreads, 0, st>>>(a.dw, a.db, offsets, E, m, plan.chunk, per,
                                                     C_out, dw, db);
    }
  }
  return launched();
}
