// Weighted sum of a row's expert outputs, and its gradients:
//   out[n] = res[n] + sum_s w[n][s] y[pos[n][s]],
//   dy[pos[n][s]] = w[n][s] dout[n],  dw[n][s] = <dout[n], y[pos[n][s]]>,
// in fp32, slot after slot, rounded once.  Both are bound by memory bandwidth:
// every row of y (and of dy) is touched once, in whole rows.  348,208 bf16 rows of
// 256 with two slots take 111 us forwards (540 MB, 4.8 TB/s; a large copy reaches
// 5.1) and 157 us backwards (897 MB, 5.7 TB/s).
#include <type_traits>

#include "rows.h"

namespace spc {
namespace {

constexpr int kThreads = 256;

// A lane per (row, 16-byte piece): LPR lanes a row, looping where the row is
// wider; the slots' loads are in flight together (K slots known, or one at a
// time for K = 0).
template <typename T, int LPR, int K, bool TAIL>
__global__ __launch_bounds__(kThreads) void k_combine_fwd(
    const T* __restrict__ y, int64_t m, const int32_t* __restrict__ pos,
    const float* __restrict__ weights, const T* res, T* out, int64_t n, int k, int C) {
  constexpr int VEC = Row<T>::VEC, G = kThreads / LPR;
  const int64_t r = static_cast<int64_t>(blockIdx.x) * G + threadIdx.x / LPR;
  if (r >= n) return;
  if constexpr (K > 0) {
    int64_t at[K];
    float w[K];
#pragma unroll
    for (int s = 0; s < K; ++s) {
      const int32_t p = pos[r * K + s];
      at[s] = p >= 0 && p < m ? static_cast<int64_t>(p) * C : -1;
      w[s] = weights ? weights[r * K + s] : 1.0f;
    }
    for (int64_t c = (blockIdx.y * LPR + threadIdx.x % LPR) * static_cast<int64_t>(VEC); c < C;
         c += static_cast<int64_t>(gridDim.y) * LPR * VEC) {
      float a[VEC], v[K][VEC];
#pragma unroll
      for (int i = 0; i < VEC; ++i) a[i] = 0.0f;
      if (res) load_row<T, TAIL>(res + r * C, c, C, a);
#pragma unroll
      for (int s = 0; s < K; ++s)
        if (at[s] >= 0) load_row<T, TAIL>(y + at[s], c, C, v[s]);
#pragma unroll
      for (int s = 0; s < K; ++s)
        if (at[s] >= 0) {
#pragma unroll
          for (int i = 0; i < VEC; ++i) a[i] += w[s] * v[s][i];
        }
      store_row<T, TAIL>(out + r * C, c, C, a);
    }
  } else {
    for (int64_t c = (blockIdx.y * LPR + threadIdx.x % LPR) * static_cast<int64_t>(VEC); c < C;
         c += static_cast<int64_t>(gridDim.y) * LPR * VEC) {
      float a[VEC];
#pragma unroll
      for (int i = 0; i < VEC; ++i) a[i] = 0.0f;
      if (res) load_row<T, TAIL>(res + r * C, c, C, a);
      for (int s = 0; s < k; ++s) {
        const int32_t p = pos[r * k + s];
        if (p < 0 || p >= m) continue;
        const float w = weights ? weights[r * k + s] : 1.0f;
        float v[VEC];
        load_row<T, TAIL>(y + static_cast<int64_t>(p) * C, c, C, v);
#pragma unroll
        for (int i = 0; i < VEC; ++i) a[i] += w * v[i];
      }
      store_row<T, TAIL>(out + r * C, c, C, a);
    }
  }
}

// Workgroups from first_zero on clear the positions no row refers to.
template <typename T>
__device__ void zero_tail(T* dy, int64_t m, const int32_t* count, int C, int64_t block,
                          int64_t blocks) {
  int64_t from = count ? *count : m;
  from = (from < 0 ? 0 : from > m ? m : from) * C;
  const int64_t end = m * C;
  for (int64_t i = from + block * kThreads + threadIdx.x; i < end; i += blocks * kThreads)
    dy[i] = Row<T>::put(0.0f);
}

// The gradient: a row's dout is read once for all its slots where those are known to the
// compiler, else once a slot, from the caches but for the first (696,416 bf16 positions of
// 256 in random order: 4 slots 187 us, 8 slots 172, 3 slots 177).
template <typename T, int LPR, int K, bool TAIL>
__global__ __launch_bounds__(kThreads) void k_combine_bwd(
    const T* __restrict__ dout, const T* __restrict__ y, const int32_t* __restrict__ pos,
    const float* __restrict__ weights, const int32_t* __restrict__ count, T* __restrict__ dy,
    float* __restrict__ dweights, int64_t m, int64_t n, int k, int C, uint32_t first_zero) {
  constexpr int VEC = Row<T>::VEC, G = kThreads / LPR;
  if (blockIdx.x >= first_zero)
    return zero_tail(dy, m, count, C, blockIdx.x - first_zero, gridDim.x - first_zero);
  const int64_t r = static_cast<int64_t>(blockIdx.x) * G + threadIdx.x / LPR;
  if (r >= n) return;                              // (whole groups of lanes)
  const int lane = threadIdx.x % LPR;
  constexpr int KS = K > 0 ? K : 1;
  for (int s0 = 0; s0 < k; s0 += KS) {
    int64_t at[KS];
    float w[KS], dot[KS];
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const int32_t p = pos[r * k + s0 + s];
      at[s] = p >= 0 && p < m ? static_cast<int64_t>(p) * C : -1;
      w[s] = weights ? weights[r * k + s0 + s] : 1.0f;
      dot[s] = 0.0f;
    }
    for (int64_t c = static_cast<int64_t>(lane) * VEC; c < C; c += LPR * VEC) {
      float d[VEC], v[KS][VEC];
      load_row<T, TAIL>(dout + r * C, c, C, d);
      if (dweights) {
#pragma unroll
        for (int s = 0; s < KS; ++s)
          if (at[s] >= 0) load_row<T, TAIL>(y + at[s], c, C, v[s]);
      }
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        if (at[s] < 0) continue;
        float o[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) o[i] = w[s] * d[i];
        store_row<T, TAIL>(dy + at[s], c, C, o);
        if (dweights) {
#pragma unroll
          for (int i = 0; i < VEC; ++i) dot[s] += d[i] * v[s][i];
        }
      }
    }
    if (dweights) {
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const float t = group_sum<LPR>(dot[s]);
        if (lane == 0) dweights[r * k + s0 + s] = at[s] >= 0 ? t : 0.0f;
      }
    }
  }
}

struct Fwd {
  const void* y;
  int64_t m;
  const int32_t* pos;
  const float* weights;
  const void* res;
  void* out;
  int64_t n;
  int k, C;
  hipStream_t st;
};
template <typename T, int LPR, int K, bool TAIL> int fwd_run(const Fwd& a) {
  const int64_t blocks = (a.n + kThreads / LPR - 1) / (kThreads / LPR);
  if (!grid_fits(blocks, kThreads)) return SPCONV_EINVAL;
  const uint32_t bx = static_cast<uint32_t>(blocks);
  // few rows: their columns over more workgroups
  const int64_t strips = (a.C + LPR * Row<T>::VEC - 1ll) / (LPR * Row<T>::VEC);
  const uint32_t by = bx >= 256 ? 1 : static_cast<uint32_t>(strips < 64 ? strips : 64);
  k_combine_fwd<T, LPR, K, TAIL><<<dim3(bx, by), kThreads, 0, a.st>>>(
      static_cast<const T*>(a.y), a.m, a.pos, a.weights, static_cast<const T*>(a.res),
      static_cast<T*>(a.out), a.n, a.k, a.C);
  return launched();
}
struct Bwd {
  const void *dout, *y;
  const int32_t* pos;
  const float* weights;
  const int32_t* count;
  void* dy;
  float* dweights;
  int64_t m, n;
  int k, C;
  hipStream_t st;
};
template <typename T, int LPR, int K, bool TAIL> int bwd_run(const Bwd& a) {
  const int64_t blocks = (a.n + kThreads / LPR - 1) / (kThreads / LPR);
  if (!grid_fits(blocks + 64, kThreads)) return SPCONV_EINVAL;
  const uint32_t bx = static_cast<uint32_t>(blocks);
  // the tail is empty, or what closed experts left: a few workgroups
  const uint32_t bz = a.count && a.m ? 64 : 0;
  if (bx + bz == 0) return SPCONV_OK;
  k_combine_bwd<T, LPR, K, TAIL><<<bx + bz, kThreads, 0, a.st>>>(
      static_cast<const T*>(a.dout), static_cast<const T*>(a.y), a.pos, a.weights, a.count,
      static_cast<T*>(a.dy), a.dweights, a.m, a.n, a.k, a.C, bx);
  return launched();
}

// LPR: the lanes a row fills, up to a wave.  Slots: 1, 2 and 4 known to the
// compiler, others one at a time.
template <typename T, int LPR, bool TAIL, typename A> int by_slots(const A& a) {
  constexpr bool kFwd = __is_same(A, Fwd);
  auto go = [&](auto kc) {
    if constexpr (kFwd) return fwd_run<T, LPR, kc.value, TAIL>(a);
    else return bwd_run<T, LPR, kc.value, TAIL>(a);
  };
  if (a.k == 1) return go(std::integral_constant<int, 1>{});
  if (a.k == 2) return go(std::integral_constant<int, 2>{});
  if (a.k == 4) return go(std::integral_constant<int, 4>{});
  return go(std::integral_constant<int, 0>{});
}
template <typename T, bool TAIL, typename A> int by_width(const A& a) {
  const int64_t pieces = (a.C + Row<T>::VEC - 1ll) / Row<T>::VEC;
  if (pieces <= 4) return by_slots<T, 4, TAIL>(a);
  if (pieces <= 8) return by_slots<T, 8, TAIL>(a);
  if (pieces <= 16) return by_slots<T, 16, TAIL>(a);
  if (pieces <= 32) return by_slots<T, 32, TAIL>(a);
  return by_slots<T, 64, TAIL>(a);
}
template <typename A> int by_type(int dt, const A& a) {
  if (dt == SPCONV_BF16)
    return a.C % 8 ? by_width<bf16_t, true>(a) : by_width<bf16_t, false>(a);
  return a.C % 4 ? by_width<float, true>(a) : by_width<float, false>(a);
}

bool sizes_ok(int dt, int64_t m, int64_t n, int k, int C) {
  return dtype_ok(dt) && rows_ok(m) && rows_ok(n) && k >= 1 && k <= SPCONV_ROUTE_MAX_SLOTS &&
         C >= 1;
}

}  // namespace
}  // namespace spc

using namespace spc;

extern "C" int spconv_combine_forward(int dt, const void* y, int64_t m, const int32_t* pos,
                                      const float* weights, const void* residual, void* out,
                                      int64_t n, int k, int C, void* stream) {
  if (!sizes_ok(dt, m, n, k, C)) return SPCONV_EINVAL;
  const size_t e = elem_bytes(dt);
  if (!ptr_ok(y, m, e) || !ptr_ok(pos, n, 4) || !aligned_to(weights, 4) ||
      !aligned_to(residual, e) || !ptr_ok(out, n, e))
    return SPCONV_EINVAL;
  if (n == 0) return SPCONV_OK;
  return by_type(dt, Fwd{y, m, pos, weights, residual, out, n, k, C,
                         static_cast<hipStream_t>(stream)});
}

extern "C" int spconv_combine_backward(int dt, const void* dout, const void* y, const int32_t* pos,
                                       const float* weights, const int32_t* count, void* dy,
                                       float* dweights, int64_t m, int64_t n, int k, int C,
                                       void* stream) {
  if (!sizes_ok(dt, m, n, k, C)) return SPCONV_EINVAL;
  const size_t e = elem_bytes(dt);
  if (!ptr_ok(dout, n, e) || !ptr_ok(y, dweights ? m : 0, e) || !ptr_ok(pos, n, 4) ||
      !aligned_to(weights, 4) || !aligned_to(count, 4) || !ptr_ok(dy, m, e) ||
      !aligned_to(dweights, 4))
    return SPCONV_EINVAL;
  if (n == 0 && m == 0) return SPCONV_OK;
  return by_type(dt, Bwd{dout, y, pos, weights, count, dy, dweights, m, n, k, C,
                         static_cast<hipStream_t>(stream)});
}
