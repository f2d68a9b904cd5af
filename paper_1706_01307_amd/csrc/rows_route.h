// Shared building blocks of the routings: the order of scores, and the (row, slot) pairs
// that a first kernel has chosen put in order by expert without atomics that decide an order.
#pragma once

#include "rows.h"

namespace spc {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kMaxE = SPCONV_ROUTE_MAX_EXPERTS;
constexpr int kMaxK = SPCONV_ROUTE_MAX_SLOTS;
constexpr int kPairs = 2048;           // pairs a workgroup ranks at most
// Counts that k_route_place adds up itself, rather than in a launch of k_route_scan
// (30,000 rows to 2 of 16, 7,504 counts: 20.2 -> 17.8 us, captured 16.7 -> 15.0; with
// 15,008 counts and four loads a lane in flight, captured 17.4 -> 21.2).
constexpr int kSumCounts = 8192;

// Rows a workgroup takes: a power of two, at most 256 (one row a lane).
__host__ __device__ inline int rows_per_block(int64_t n, int E, int k) {
  int r = 256;
  while (r * k > kPairs) r /= 2;
  // so few that one workgroup is done sooner than two more launches begin
  if (n <= r && n * E <= 16384) return r;
  // as long as there are fewer workgroups than compute units
  while (r > 32 && (n + r - 1) / r < 256) r /= 2;
  return r;
}

// A logit's order as an unsigned number: larger is larger, -0 equals +0, every
// NaN is the largest.  0 is below -infinity (kNone).
constexpr uint32_t kNone = 0x007fffffu;            // the order of -infinity
__device__ __forceinline__ uint32_t order_of(float v) {
  if (v != v) return 0xffffffffu;
  const uint32_t u = __float_as_uint(v + 0.0f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t o) {
  return __uint_as_float(o == 0xffffffffu ? 0x7fc00000u : o & 0x80000000u ? o & 0x7fffffffu : ~o);
}

// The largest (order, lowest column) of the group's lanes.
template <int STEP> __device__ __forceinline__ void best_step(uint32_t& o, uint32_t& c) {
  const uint32_t o2 = lane_other<STEP>(o), c2 = lane_other<STEP>(c);
  const bool take = o2 > o || (o2 == o && c2 < c);
  o = take ? o2 : o;
  c = take ? c2 : c;
}
template <int LPR> __device__ __forceinline__ void group_best(uint32_t& o, uint32_t& c) {
  if constexpr (LPR > 1) best_step<1>(o, c);
  if constexpr (LPR > 2) best_step<2>(o, c);
  if constexpr (LPR > 4) best_step<4>(o, c);
  if constexpr (LPR > 8) best_step<8>(o, c);
  if constexpr (LPR > 16) {
    const auto a = __builtin_amdgcn_permlane16_swap(o, o, false, false);
    const auto b = __builtin_amdgcn_permlane16_swap(c, c, false, false);
    const bool take = a[1] > a[0] || (a[1] == a[0] && b[1] < b[0]);
    o = take ? a[1] : a[0];
    c = take ? b[1] : b[0];
  }
  if constexpr (LPR > 32) {
    const auto a = __builtin_amdgcn_permlane32_swap(o, o, false, false);
    const auto b = __builtin_amdgcn_permlane32_swap(c, c, false, false);
    const bool take = a[1] > a[0] || (a[1] == a[0] && b[1] < b[0]);
    o = take ? a[1] : a[0];
    c = take ? b[1] : b[0];
  }
}

// The sum over a whole wave's lanes before this one.
__device__ __forceinline__ int32_t wave_exclusive(int32_t v, int32_t* total) {
  int32_t s = v;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int32_t o = __shfl_up(s, d, 64);
    if (static_cast<int>(threadIdx.x & 63) >= d) s += o;
  }
  *total = __shfl(s, 63, 64);
  return s - v;
}

// Exclusive running sums of v[0..E) in place, E <= kMaxE; the whole workgroup
// calls it.  Returns the total.
__device__ int32_t block_scan(int32_t* v, int E, int32_t* s_wave) {
  constexpr int PER = kMaxE / kThreads;
  const int wave = threadIdx.x >> 6;
  int32_t a[PER], sum = 0;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int e = threadIdx.x * PER + i;
    a[i] = e < E ? v[e] : 0;
    sum += a[i];
  }
  int32_t total;
  int32_t base = wave_exclusive(sum, &total);
  if ((threadIdx.x & 63) == 0) s_wave[wave] = total;
  __syncthreads();
  int32_t all = 0;
#pragma unroll
  for (int q = 0; q < kWaves; ++q) {
    if (q < wave) base += s_wave[q];
    all += s_wave[q];
  }
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int e = threadIdx.x * PER + i;
    if (e < E) v[e] = base;
    base += a[i];
  }
  __syncthreads();
  return all;
}

// The second half of a routing's first kernel, once s_expert and s_weight hold the `nrow` rows
// from row0: they are written out, and every pair is ranked among the workgroup's own of its
// expert; the counts are left to k_route_place, or, with one workgroup, everything is done.
__device__ __forceinline__ void rank_pairs(
    int64_t n, int E, int k, int64_t row0, int nrow, const int16_t* s_expert,
    const float* s_weight, int32_t (&s_count)[kWaves][kMaxE], int32_t* s_start, int32_t* s_wave,
    int32_t* __restrict__ experts, float* __restrict__ weights, int32_t* __restrict__ offsets,
    int32_t* __restrict__ rows, int32_t* __restrict__ pos, int32_t* __restrict__ counts) {
  __syncthreads();
  const int npair = nrow * k, wave = threadIdx.x >> 6, wl = threadIdx.x & 63;
  for (int p = threadIdx.x; p < npair; p += kThreads) {
    experts[row0 * k + p] = s_expert[p];
    weights[row0 * k + p] = s_weight[p];
  }

  // Ranks: each wave takes a run of the pairs, counts it per expert, and then
  // numbers it 64 pairs at a time from where the runs before it end.
  const int run = (npair + kWaves * 64 - 1) / (kWaves * 64) * 64;
  const int p0 = wave * run, p1 = p0 + run < npair ? p0 + run : npair;
  for (int p = p0 + wl; p < p1; p += 64) {
    const int e = s_expert[p];
    if (e >= 0) atomicAdd(&s_count[wave][e], 1);   // (a count: no order in it)
  }
  __syncthreads();
  const bool single = gridDim.x == 1;
  for (int e = threadIdx.x; e < E; e += kThreads) {
    int32_t a = 0;
#pragma unroll
    for (int q = 0; q < kWaves; ++q) {
      const int32_t c = s_count[q][e];
      s_count[q][e] = a;
      a += c;
    }
    s_start[e] = a;
    if (!single) counts[static_cast<int64_t>(e) * gridDim.x + blockIdx.x] = a;
  }
  int32_t total = 0;
  if (single) {
    total = block_scan(s_start, E, s_wave);
    for (int e = threadIdx.x; e < E; e += kThreads) offsets[e] = s_start[e];
    if (threadIdx.x == 0) offsets[E] = total;
  }
  __syncthreads();
  int ebits = 0;
  while ((1 << ebits) < E) ++ebits;
  for (int b = p0; b < p1; b += 64) {              // (uniform over the wave)
    const int p = b + wl;
    const int e = p < p1 ? s_expert[p] : -1;
    uint64_t same = __ballot(e >= 0);
    for (int t = 0; t < ebits; ++t) {
      const uint64_t m = __ballot((e >> t) & 1);
      same &= (e >> t) & 1 ? m : ~m;
    }
    if (e >= 0) {
      const int before = __popcll(same & ((1ull << wl) - 1));
      const int32_t rank = s_count[wave][e] + before;
      const int64_t at = row0 * k + p;
      if (single) {
        const int32_t where = s_start[e] + rank;
        pos[at] = where;
        rows[where] = static_cast<int32_t>(row0 + p / k);
      } else {
        pos[at] = rank;                            // k_route_place adds the starts
      }
    } else if (p < p1) {
      pos[row0 * k + p] = -1;
    }
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    // the last of each expert's lanes moves its count on
    if (e >= 0 && (same >> wl) == 1ull) s_count[wave][e] += __popcll(same);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
  if (single)
    for (int64_t p = total + threadIdx.x; p < n * k; p += kThreads) rows[p] = -1;
}

// A workgroup per expert: exclusive running sums of its counts over the
// workgroups, in place; the total behind them.
__global__ __launch_bounds__(1024) void k_route_scan(int32_t* __restrict__ counts, int nblk,
                                                     int32_t* __restrict__ totals) {
  __shared__ int32_t s_wave[16];
  int32_t* c = counts + static_cast<int64_t>(blockIdx.x) * nblk;
  const int wave = threadIdx.x >> 6;
  int32_t carry = 0;
  for (int b = 0; b < nblk; b += 1024) {
    const int i = b + threadIdx.x;
    const int32_t v = i < nblk ? c[i] : 0;
    int32_t total;
    int32_t ex = wave_exclusive(v, &total);
    if ((threadIdx.x & 63) == 0) s_wave[wave] = total;
    __syncthreads();
    int32_t all = 0;
#pragma unroll
    for (int q = 0; q < 16; ++q) {
      if (q < wave) ex += s_wave[q];
      all += s_wave[q];
    }
    if (i < nblk) c[i] = carry + ex;
    carry += all;
    __syncthreads();
  }
  if (threadIdx.x == 0) totals[blockIdx.x] = carry;
}

// SUM: `counts` are k_route's, and every workgroup adds up those before its own and
// all of them, four experts a wave in turn; else they are k_route_scan's running sums.
template <bool SUM>
__global__ __launch_bounds__(kThreads) void k_route_place(
    const int32_t* __restrict__ experts, const int32_t* __restrict__ counts,
    const int32_t* __restrict__ totals, int64_t n, int E, int k, int rows_blk,
    int32_t* __restrict__ offsets, int32_t* __restrict__ rows, int32_t* __restrict__ pos) {
  __shared__ int32_t s_start[kMaxE], s_before[SUM ? kMaxE : 1], s_wave[kWaves];
  const int nblk = gridDim.x, blk = blockIdx.x;
  if constexpr (SUM) {
    constexpr int N = 4, U = 4;                    // experts, counts of each, in flight together
    for (int e0 = (threadIdx.x >> 6) * N; e0 < E; e0 += kWaves * N) {
      int32_t before[N] = {}, all[N] = {};
      for (int b0 = threadIdx.x & 63; b0 < nblk; b0 += 64 * U) {
        int32_t v[U][N];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int i = 0; i < N; ++i) {
            const int e = e0 + i < E ? e0 + i : E - 1, b = b0 + 64 * u;
            v[u][i] = counts[static_cast<int64_t>(e) * nblk + (b < nblk ? b : b0)];
          }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int i = 0; i < N; ++i) {
            all[i] += b0 + 64 * u < nblk ? v[u][i] : 0;
            before[i] += b0 + 64 * u < blk ? v[u][i] : 0;
          }
      }
#pragma unroll
      for (int d = 1; d < 64; d *= 2)
#pragma unroll
        for (int i = 0; i < N; ++i) {
          all[i] += __shfl_xor(all[i], d, 64);
          before[i] += __shfl_xor(before[i], d, 64);
        }
#pragma unroll
      for (int i = 0; i < N; ++i)
        if ((threadIdx.x & 63) == i && e0 + i < E) {
          s_start[e0 + i] = all[i];
          s_before[e0 + i] = before[i];
        }
    }
  } else {
    for (int e = threadIdx.x; e < E; e += kThreads) s_start[e] = totals[e];
  }
  const int32_t total = block_scan(s_start, E, s_wave);
  if (blk == 0) {
    for (int e = threadIdx.x; e < E; e += kThreads) offsets[e] = s_start[e];
    if (threadIdx.x == 0) offsets[E] = total;
    __syncthreads();
  }
  for (int e = threadIdx.x; e < E; e += kThreads)
    s_start[e] += SUM ? s_before[e] : counts[static_cast<int64_t>(e) * nblk + blk];
  __syncthreads();
  const int64_t row0 = static_cast<int64_t>(blockIdx.x) * rows_blk;
  const int64_t end = (row0 + rows_blk < n ? row0 + rows_blk : n) * k;
  for (int64_t p = row0 * k + threadIdx.x; p < end; p += kThreads) {
    const int32_t e = experts[p];
    if (e < 0) continue;
    const int32_t where = s_start[e] + pos[p];
    pos[p] = where;
    rows[where] = static_cast<int32_t>(row0 + static_cast<int32_t>(p - row0 * k) / k);
  }
  for (int64_t p = total + static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; p < n * k;
       p += static_cast<int64_t>(gridDim.x) * kThreads)
    rows[p] = -1;
}

// The launches behind the one that leaves the counts of `nblk` > 1 workgroups.
inline void place_pairs(const int32_t* experts, int32_t* counts, int nblk, int64_t n, int E, int k,
                        int rb, int32_t* offsets, int32_t* rows, int32_t* pos, hipStream_t st) {
  int32_t* totals = counts + static_cast<int64_t>(nblk) * E;
  if (static_cast<int64_t>(nblk) * E <= kSumCounts) {
    k_route_place<true><<<nblk, kThreads, 0, st>>>(experts, counts, nullptr, n, E, k, rb, offsets,
                                                  rows, pos);
  } else {
    k_route_scan<<<E, 1024, 0, st>>>(counts, nblk, totals);
    k_route_place<false><<<nblk, kThreads, 0, st>>>(experts, counts, totals, n, E, k, rb, offsets,
                                                   rows, pos);
  }
}

inline bool sizes_ok(int64_t n, int E, int k) {
  return rows_ok(n) && E >= 1 && E <= kMaxE && k >= 1 && k <= kMaxK && k <= E && rows_ok(n * k);
}
// The workspace of a call: the workgroups' counts, and their totals.
inline size_t counts_bytes(int64_t n, int E, int k) {
  const int rb = rows_per_block(n, E, k);
  const int64_t nblk = (n + rb - 1) / rb;
  return nblk > 1 ? static_cast<size_t>((nblk + 1) * E) * sizeof(int32_t) : 0;
}

}  // namespace
}  // namespace spc
