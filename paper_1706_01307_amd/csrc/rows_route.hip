// Routing: the k largest logits of every row, their softmax weights, and the
// (row, slot) pairs grouped by expert in a stable order, without atomics that
// decide an order.
//
//   k_route        a group of lanes per row picks the experts; the workgroup
//                  ranks its own pairs per expert and leaves its counts;
//   k_route_scan   per expert, the counts' running sums over the workgroups (few
//                  counts are left to k_route_place);
//   k_route_place  every pair's position: its expert's start + its
//                  workgroup's start + its rank.
// Where one workgroup has every row, the first launch does it all.
//
// 348,208 rows of 64 fp32 logits to 2 each: 30 + 4 + 5 us, where the bytes alone
// would take 20: k_route is bound by the k dependent searches of a row (compares and
// lane exchanges keep the vector ALU for 70 % of the cycles it has work), the other two
// are short.
#include <cmath>

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

// LPR lanes hold a row of at most LPR * NV * VEC logits.
template <typename T, int LPR, int NV, bool TAIL>
__global__ __launch_bounds__(kThreads) void k_route(
    const T* __restrict__ logits, int64_t n, int E, int k, int normalize, int rows_blk,
    int32_t* __restrict__ experts, float* __restrict__ weights, int32_t* __restrict__ offsets,
    int32_t* __restrict__ rows, int32_t* __restrict__ pos, int32_t* __restrict__ counts) {
  constexpr int VEC = Row<T>::VEC, G = kThreads / LPR;
  __shared__ int16_t s_expert[kPairs];
  __shared__ float s_weight[kPairs];
  __shared__ int32_t s_count[kWaves][kMaxE];       // running counts of the waves' runs of pairs
  __shared__ int32_t s_start[kMaxE], s_wave[kWaves];
  const int lane = threadIdx.x % LPR;
  const int64_t row0 = static_cast<int64_t>(blockIdx.x) * rows_blk;
  const int nrow = static_cast<int>(n - row0 < rows_blk ? n - row0 : rows_blk);
  for (int e = threadIdx.x; e < E; e += kThreads)
#pragma unroll
    for (int q = 0; q < kWaves; ++q) s_count[q][e] = 0;

  // UR rows of a group at a time, for their chains of lane exchanges to overlap, and
  // the next ones' logits on their way meanwhile (a group's lanes stay together).
  constexpr int UR = NV == 1 ? 2 : 1;
  float next[UR][NV][VEC];
  auto request = [&](int q0) {
#pragma unroll
    for (int u = 0; u < UR; ++u)
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const int q = q0 + G * u, c = (lane + LPR * j) * VEC;
        if (q < nrow && c < E) load_row<T, TAIL>(logits + (row0 + q) * E, c, E, next[u][j]);
      }
  };
  request(threadIdx.x / LPR);
  for (int q0 = threadIdx.x / LPR; q0 < nrow; q0 += G * UR) {
    uint32_t o[UR][NV][VEC];
    float top[UR], sum[UR];
#pragma unroll
    for (int u = 0; u < UR; ++u) {
      sum[u] = 0.0f;
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < VEC; ++i)
          o[u][j][i] = (lane + LPR * j) * VEC + i < E ? order_of(next[u][j][i]) : 0u;
    }
    request(q0 + G * UR);
    for (int s = 0; s < k; ++s) {
      uint32_t bo[UR], bc[UR];
#pragma unroll
      for (int u = 0; u < UR; ++u) {
        bo[u] = 0;
        bc[u] = 0xffffffffu;
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
          for (int i = 0; i < VEC; ++i)
            if (o[u][j][i] > bo[u]) {              // ascending columns: the lowest of equals
              bo[u] = o[u][j][i];
              bc[u] = (lane + LPR * j) * VEC + i;
            }
        group_best<LPR>(bo[u], bc[u]);
      }
#pragma unroll
      for (int u = 0; u < UR; ++u) {
        const bool some = bo[u] > kNone;
        const float v = value_of(bo[u]);
        if (s == 0) {
          top[u] = some ? v : 0.0f;
          if (!normalize) {
            // the whole row's sum, before anything is taken out of it
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
              for (int i = 0; i < VEC; ++i)
                if (o[u][j][i]) sum[u] += expf(value_of(o[u][j][i]) - top[u]);
            sum[u] = group_sum<LPR>(sum[u]);
          }
        }
        const float w = some ? expf(v - top[u]) : 0.0f;
        if (normalize) sum[u] += w;
        const int q = q0 + G * u;
        if (lane == s % LPR && q < nrow) {
          s_expert[q * k + s] = static_cast<int16_t>(some ? static_cast<int32_t>(bc[u]) : -1);
          s_weight[q * k + s] = w;
        }
        // take it out
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
          for (int i = 0; i < VEC; ++i)
            if (static_cast<uint32_t>((lane + LPR * j) * VEC + i) == bc[u]) o[u][j][i] = 0u;
      }
    }
    // (each lane divides the slots it wrote)
#pragma unroll
    for (int u = 0; u < UR; ++u) {
      const int q = q0 + G * u;
      for (int s = lane; s < k && q < nrow; s += LPR)
        if (s_expert[q * k + s] >= 0) s_weight[q * k + s] /= sum[u];
    }
  }
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

// The gradient: every lane sums the row's slots itself (they are the same
// addresses for the whole group), then finds its columns among them.
template <typename T, int LPR, int NV, bool TAIL>
__global__ __launch_bounds__(kThreads) void k_route_bwd(
    const float* __restrict__ dweights, const T* __restrict__ logits,
    const int32_t* __restrict__ experts, const float* __restrict__ weights, int64_t n, int E,
    int k, int normalize, T* __restrict__ dlogits) {
  constexpr int VEC = Row<T>::VEC, G = kThreads / LPR;
  const int lane = threadIdx.x % LPR;
  const int64_t r = static_cast<int64_t>(blockIdx.x) * G + threadIdx.x / LPR;
  if (r >= n) return;
  float v[NV][VEC];
  float inv = 0.0f;
  if (!normalize) {
    float top = -INFINITY, sum = 0.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (lane + LPR * j) * VEC;
#pragma unroll
      for (int i = 0; i < VEC; ++i) v[j][i] = -INFINITY;
      if (c < E) load_row<T, TAIL>(logits + r * E, c, E, v[j]);
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        if (c + i >= E) v[j][i] = -INFINITY;
        top = v[j][i] > top || v[j][i] != v[j][i] ? v[j][i] : top;
      }
    }
    top = group_reduce<LPR>(top, [](float a, float b) { return b > a || b != b ? b : a; });
    if (top == -INFINITY) top = 0.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        v[j][i] = expf(v[j][i] - top);
        sum += v[j][i];
      }
    sum = group_sum<LPR>(sum);
    inv = sum == 0.0f ? 0.0f : 1.0f / sum;         // (a row that is all closed)
  }
  float dot = 0.0f;
  for (int s = 0; s < k; ++s)
    if (experts[r * k + s] >= 0) dot += weights[r * k + s] * dweights[r * k + s];
  float g[NV][VEC];
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int i = 0; i < VEC; ++i) g[j][i] = normalize ? 0.0f : -(v[j][i] * inv) * dot;
  for (int s = 0; s < k; ++s) {
    const int32_t e = experts[r * k + s];
    if (e < 0) continue;
    const float d = weights[r * k + s] * (normalize ? dweights[r * k + s] - dot
                                                    : dweights[r * k + s]);
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int i = 0; i < VEC; ++i)
        if ((lane + LPR * j) * VEC + i == e) g[j][i] += d;
  }
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int c = (lane + LPR * j) * VEC;
    if (c < E) store_row<T, TAIL>(dlogits + r * E, c, E, g[j]);
  }
}

struct Fwd {
  const void* logits;
  int64_t n;
  int E, k, normalize;
  int32_t* experts;
  float* weights;
  int32_t *offsets, *rows, *pos, *counts;
  hipStream_t st;
};
template <typename T, int LPR, int NV> int run(const Fwd& a) {
  const int rb = rows_per_block(a.n, a.E, a.k);
  const int nblk = a.n ? static_cast<int>((a.n + rb - 1) / rb) : 1;
  const T* l = static_cast<const T*>(a.logits);
  if (a.E % Row<T>::VEC)
    k_route<T, LPR, NV, true><<<nblk, kThreads, 0, a.st>>>(l, a.n, a.E, a.k, a.normalize, rb,
                                                          a.experts, a.weights, a.offsets, a.rows,
                                                          a.pos, a.counts);
  else
    k_route<T, LPR, NV, false><<<nblk, kThreads, 0, a.st>>>(l, a.n, a.E, a.k, a.normalize, rb,
                                                           a.experts, a.weights, a.offsets, a.rows,
                                                           a.pos, a.counts);
  if (nblk > 1) {
    int32_t* totals = a.counts + static_cast<int64_t>(nblk) * a.E;
    if (static_cast<int64_t>(nblk) * a.E <= kSumCounts) {
      k_route_place<true><<<nblk, kThreads, 0, a.st>>>(a.experts, a.counts, nullptr, a.n, a.E, a.k,
                                                      rb, a.offsets, a.rows, a.pos);
    } else {
      k_route_scan<<<a.E, 1024, 0, a.st>>>(a.counts, nblk, totals);
      k_route_place<false><<<nblk, kThreads, 0, a.st>>>(a.experts, a.counts, totals, a.n, a.E, a.k,
                                                       rb, a.offsets, a.rows, a.pos);
    }
  }
  return launched();
}
struct Bwd {
  const float* dweights;
  const void* logits;
  const int32_t* experts;
  const float* weights;
  int64_t n;
  int E, k, normalize;
  void* dlogits;
  hipStream_t st;
};
template <typename T, int LPR, int NV> int run(const Bwd& a) {
  const int64_t want = (a.n + kThreads / LPR - 1) / (kThreads / LPR);
  if (!grid_fits(want, kThreads)) return SPCONV_EINVAL;
  const uint32_t blocks = static_cast<uint32_t>(want);
  const T* l = static_cast<const T*>(a.logits);
  T* d = static_cast<T*>(a.dlogits);
  if (a.E % Row<T>::VEC)
    k_route_bwd<T, LPR, NV, true><<<blocks, kThreads, 0, a.st>>>(
        a.dweights, l, a.experts, a.weights, a.n, a.E, a.k, a.normalize, d);
  else
    k_route_bwd<T, LPR, NV, false><<<blocks, kThreads, 0, a.st>>>(
        a.dweights, l, a.experts, a.weights, a.n, a.E, a.k, a.normalize, d);
  return launched();
}
// Up to four pieces a lane, then more lanes: a step of the exchange between lanes
// costs a wave the same for 4 rows as for 16 (64 fp32 logits, 348,208 rows: four
// lanes a row 31 us, sixteen with a piece each 48).
template <typename T, typename A> int by_width(const A& a) {
  const int pieces = (a.E + Row<T>::VEC - 1) / Row<T>::VEC;
  if (pieces <= 1) return run<T, 1, 1>(a);
  if (pieces <= 2) return run<T, 1, 2>(a);
  if (pieces <= 4) return run<T, 1, 4>(a);
  if (pieces <= 8) return run<T, 2, 4>(a);
  if (pieces <= 16) return run<T, 4, 4>(a);
  if (pieces <= 32) return run<T, 8, 4>(a);
  if (pieces <= 64) return run<T, 16, 4>(a);
  if (pieces <= 128) return run<T, 32, 4>(a);
  if constexpr (Row<T>::VEC == 4) return run<T, 64, 4>(a);
  return SPCONV_EINVAL;                            // (not reached: E <= kMaxE)
}

bool sizes_ok(int64_t n, int E, int k) {
  return rows_ok(n) && E >= 1 && E <= kMaxE && k >= 1 && k <= kMaxK && k <= E && rows_ok(n * k);
}

}  // namespace
}  // namespace spc

using namespace spc;

extern "C" int spconv_route_workspace(int64_t n, int E, int k, size_t* bytes) {
  if (!sizes_ok(n, E, k) || !bytes) return SPCONV_EINVAL;
  const int rb = rows_per_block(n, E, k);
  const int64_t nblk = (n + rb - 1) / rb;
  *bytes = nblk > 1 ? static_cast<size_t>((nblk + 1) * E) * sizeof(int32_t) : 0;
  return SPCONV_OK;
}

extern "C" int spconv_route_forward(int dt, const void* logits, int64_t n, int E, int k,
                                    int normalize, int32_t* experts, float* weights,
                                    int32_t* offsets, int32_t* rows, int32_t* pos, void* workspace,
                                    size_t workspace_bytes, void* stream) {
  size_t need = 0;
  if (!dtype_ok(dt) || (normalize != 0 && normalize != 1) ||
      spconv_route_workspace(n, E, k, &need) != SPCONV_OK || !ptr_ok(logits, n, elem_bytes(dt)) ||
      !ptr_ok(experts, n, 4) || !ptr_ok(weights, n, 4) || !ptr_ok(offsets, 1, 4) ||
      !ptr_ok(rows, n, 4) || !ptr_ok(pos, n, 4) ||
      (need && (!workspace || !aligned_to(workspace, 16) || workspace_bytes < need)))
    return SPCONV_EINVAL;
  // (no rows: one workgroup without rows writes the offsets)
  const Fwd a{logits, n, E, k, normalize, experts, weights, offsets, rows, pos,
              static_cast<int32_t*>(workspace), static_cast<hipStream_t>(stream)};
  return dt == SPCONV_BF16 ? by_width<bf16_t>(a) : by_width<float>(a);
}

extern "C" int spconv_route_backward(int dt, const float* dweights, const void* logits,
                                     const int32_t* experts, const float* weights, int64_t n, int E,
                                     int k, int normalize, void* dlogits, void* stream) {
  if (!dtype_ok(dt) || (normalize != 0 && normalize != 1) || !sizes_ok(n, E, k) ||
      !ptr_ok(dweights, n, 4) || !ptr_ok(logits, normalize ? 0 : n, elem_bytes(dt)) ||
      !ptr_ok(experts, n, 4) || !ptr_ok(weights, n, 4) || !ptr_ok(dlogits, n, elem_bytes(dt)))
    return SPCONV_EINVAL;
  if (n == 0) return SPCONV_OK;
  const Bwd a{dweights, logits, experts, weights, n, E, k, normalize, dlogits,
              static_cast<hipStream_t>(stream)};
  return dt == SPCONV_BF16 ? by_width<bf16_t>(a) : by_width<float>(a);
}
