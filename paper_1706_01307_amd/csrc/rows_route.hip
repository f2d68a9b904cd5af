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

#include "rows_route.h"

namespace spc {
namespace {

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
  rank_pairs(n, E, k, row0, nrow, s_expert, s_weight, s_count, s_start, s_wave, experts, weights,
             offsets, rows, pos, counts);
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
  if (nblk > 1)
    place_pairs(a.experts, a.counts, nblk, a.n, a.E, a.k, rb, a.offsets, a.rows, a.pos, a.st);
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

}  // namespace
}  // namespace spc

using namespace spc;

extern "C" int spconv_route_workspace(int64_t n, int E, int k, size_t* bytes) {
  if (!sizes_ok(n, E, k) || !bytes) return SPCONV_EINVAL;
  *bytes = counts_bytes(n, E, k);
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
