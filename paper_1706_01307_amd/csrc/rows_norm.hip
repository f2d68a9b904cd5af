// Layer norm of feature rows and its gradients.
//
// One pass over the rows: a row lives in the registers of a group of lanes
// between its statistics and its output, so that memory is read and written
// once; the group's sums go over the vector ALU's lane permutations.  Both
// directions are bound by memory bandwidth: 902,504 bf16 rows of 64 take 40 us
// forwards (6.0 TB/s; a large copy reaches 5.1, less of it from the last-level
// cache) and 62 + 4 us backwards (5.7 TB/s), 87,052 fp32 rows of 145 backwards
// 31 + 4 us (5.0 TB/s).
#include <cmath>

#include "rows.h"

namespace spc {
namespace {

constexpr int kThreads = 256;

// Sums over the LPR lanes that hold a row (256: the whole workgroup).
template <int LPR> struct RowSum {
  float* s;
  int turn = 0;
  __device__ explicit RowSum(float* lds) : s(lds) {}
  __device__ float operator()(float v) {
    if constexpr (LPR <= 64) return group_sum<LPR>(v);
    return block_sum(v, s, turn++);
  }
};

// y = (x - mean) rstd gamma + beta with rstd = 1 / sqrt(mean of (x - mean)^2 + eps),
// the squares taken of x - mean (the difference of two large sums would cancel).
// A group of LPR lanes holds a row of at most LPR * NV * VEC elements: NV
// pieces of 16 bytes a lane.  The group takes UR rows at a time, their loads in
// flight together.
template <typename T, int LPR, int NV, int UR, bool TAIL>
__global__ __launch_bounds__(kThreads) void k_norm_fwd(
    const T* __restrict__ x, const float* __restrict__ gamma, const float* __restrict__ beta,
    float eps, T* __restrict__ y, float* __restrict__ mean, float* __restrict__ rstd, int64_t n,
    int C) {
  constexpr int VEC = Row<T>::VEC, G = kThreads / LPR;
  __shared__ float s_sum[8];
  RowSum<LPR> sum(s_sum);
  const int lane = threadIdx.x % LPR;
  const int64_t first = (static_cast<int64_t>(blockIdx.x) * G + threadIdx.x / LPR) * UR;
  float v[UR][NV][VEC];
#pragma unroll
  for (int u = 0; u < UR; ++u)
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (lane + LPR * j) * VEC;
#pragma unroll
      for (int i = 0; i < VEC; ++i) v[u][j][i] = 0.0f;
      if (first + u < n && c < C) load_row<T, TAIL>(x + (first + u) * C, c, C, v[u][j]);
    }
  float mu[UR], rs[UR];
#pragma unroll
  for (int u = 0; u < UR; ++u) {
    float a = 0.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int i = 0; i < VEC; ++i) a += v[u][j][i];
    mu[u] = sum(a) / C;
  }
#pragma unroll
  for (int u = 0; u < UR; ++u) {
    float a = 0.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        const int c = (lane + LPR * j) * VEC + i;
        v[u][j][i] -= mu[u];
        if (c < C) a += v[u][j][i] * v[u][j][i];
      }
    rs[u] = 1.0f / sqrtf(sum(a) / C + eps);
  }
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int c = (lane + LPR * j) * VEC;
    if (c >= C) continue;
    float g[VEC], b[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) g[i] = 1.0f, b[i] = 0.0f;
    if (gamma) load_f32<VEC, TAIL>(gamma, c, C, g);
    if (beta) load_f32<VEC, TAIL>(beta, c, C, b);
#pragma unroll
    for (int u = 0; u < UR; ++u) {
      if (first + u >= n) break;
      float o[VEC];
#pragma unroll
      for (int i = 0; i < VEC; ++i) o[i] = v[u][j][i] * rs[u] * g[i] + b[i];
      store_row<T, TAIL>(y + (first + u) * C, c, C, o);
    }
  }
  if (mean && lane == 0)
#pragma unroll
    for (int u = 0; u < UR; ++u)
      if (first + u < n) {
        mean[first + u] = mu[u];
        rstd[first + u] = rs[u];
      }
}

// Rows too wide for a workgroup's registers: a workgroup per row, which it
// reads three times (twice from the caches).
template <typename T>
__global__ __launch_bounds__(kThreads) void k_norm_fwd_wide(
    const T* __restrict__ x, const float* __restrict__ gamma, const float* __restrict__ beta,
    float eps, T* __restrict__ y, float* __restrict__ mean, float* __restrict__ rstd, int C) {
  constexpr int VEC = Row<T>::VEC;
  __shared__ float s_sum[8];
  const int64_t r = blockIdx.x;
  x += r * C;
  y += r * C;
  const int64_t step = kThreads * VEC, c0 = threadIdx.x * VEC;
  float a = 0.0f, v[VEC];
  for (int64_t c = c0; c < C; c += step) {
    load_row<T, true>(x, c, C, v);
#pragma unroll
    for (int i = 0; i < VEC; ++i) a += v[i];
  }
  const float mu = block_sum(a, s_sum, 0) / C;
  a = 0.0f;
  for (int64_t c = c0; c < C; c += step) {
    load_row<T, true>(x, c, C, v);
#pragma unroll
    for (int i = 0; i < VEC; ++i)
      if (c + i < C) a += (v[i] - mu) * (v[i] - mu);
  }
  const float rs = 1.0f / sqrtf(block_sum(a, s_sum, 1) / C + eps);
  for (int64_t c = c0; c < C; c += step) {
    float g[VEC], b[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) g[i] = 1.0f, b[i] = 0.0f;
    if (gamma) load_f32<VEC, true>(gamma, c, C, g);
    if (beta) load_f32<VEC, true>(beta, c, C, b);
    load_row<T, true>(x, c, C, v);
#pragma unroll
    for (int i = 0; i < VEC; ++i) v[i] = (v[i] - mu) * rs * g[i] + b[i];
    store_row<T, true>(y, c, C, v);
  }
  if (mean && threadIdx.x == 0) {
    mean[r] = mu;
    rstd[r] = rs;
  }
}

// The gradient, rows held as above: with z = (x - mean) rstd and d = gamma dy,
// dx = rstd (d - mean of d - z mean of d z).  With PARAM, a lane keeps its columns' sums
// of dy z and dy over the rows its group takes (every gridDim.x * G-th batch of
// UR rows); the groups' sums are added through LDS in group order and leave as
// the workgroup's row of `part` ([2][C]), which k_norm_parts adds up.
template <typename T, int LPR, int NV, int UR, bool TAIL, bool PARAM>
__global__ __launch_bounds__(kThreads) void k_norm_bwd(
    const T* __restrict__ dy, const T* __restrict__ x, const float* __restrict__ mean,
    const float* __restrict__ rstd, const float* __restrict__ gamma, T* __restrict__ dx,
    float* __restrict__ part, int64_t n, int C) {
  constexpr int VEC = Row<T>::VEC, G = kThreads / LPR;
  __shared__ float s_sum[8];
  RowSum<LPR> sum(s_sum);
  const int lane = threadIdx.x % LPR, group = threadIdx.x / LPR;
  float g[NV][VEC];
  float ag[PARAM ? NV : 1][VEC], ab[PARAM ? NV : 1][VEC];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int c = (lane + LPR * j) * VEC;
#pragma unroll
    for (int i = 0; i < VEC; ++i) g[j][i] = 1.0f;
    if (gamma && c < C) load_f32<VEC, TAIL>(gamma, c, C, g[j]);
    if constexpr (PARAM) {
#pragma unroll
      for (int i = 0; i < VEC; ++i) ag[j][i] = ab[j][i] = 0.0f;
    }
  }
  const int64_t stride = static_cast<int64_t>(gridDim.x) * G * UR;
  // uniform over the workgroup (the sums have barriers)
  for (int64_t base = static_cast<int64_t>(blockIdx.x) * G * UR; base < n; base += stride) {
    const int64_t first = base + static_cast<int64_t>(group) * UR;
    float d[UR][NV][VEC], z[UR][NV][VEC];
    float mu[UR], rs[UR];
#pragma unroll
    for (int u = 0; u < UR; ++u) {
      const bool live = first + u < n;
      mu[u] = live ? mean[first + u] : 0.0f;
      rs[u] = live ? rstd[first + u] : 0.0f;
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const int c = (lane + LPR * j) * VEC;
#pragma unroll
        for (int i = 0; i < VEC; ++i) d[u][j][i] = z[u][j][i] = 0.0f;
        if (live && c < C) {
          load_row<T, TAIL>(dy + (first + u) * C, c, C, d[u][j]);
          load_row<T, TAIL>(x + (first + u) * C, c, C, z[u][j]);
        }
      }
    }
#pragma unroll
    for (int u = 0; u < UR; ++u) {
      float a = 0.0f, b = 0.0f;
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          const int c = (lane + LPR * j) * VEC + i;
          // past the row's end d is zero; z must not be (x - mean) there
          z[u][j][i] = c < C ? (z[u][j][i] - mu[u]) * rs[u] : 0.0f;
          if constexpr (PARAM) {
            ag[j][i] += d[u][j][i] * z[u][j][i];
            ab[j][i] += d[u][j][i];
          }
          d[u][j][i] *= g[j][i];
          a += d[u][j][i];
          b += d[u][j][i] * z[u][j][i];
        }
      const float ma = sum(a) / C, mb = sum(b) / C;
      if (first + u < n) {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
          const int c = (lane + LPR * j) * VEC;
          if (c >= C) continue;
          float o[VEC];
#pragma unroll
          for (int i = 0; i < VEC; ++i) o[i] = rs[u] * (d[u][j][i] - ma - z[u][j][i] * mb);
          store_row<T, TAIL>(dx + (first + u) * C, c, C, o);
        }
      }
    }
  }
  if constexpr (PARAM) {
    float* out = part + static_cast<int64_t>(blockIdx.x) * 2 * C;
    __shared__ float s_part[G > 1 ? 2 * kThreads * VEC : 1];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      if constexpr (G == 1) {
        const int c = (lane + LPR * j) * VEC;
#pragma unroll
        for (int i = 0; i < VEC; ++i)
          if (c + i < C) {
            out[c + i] = ag[j][i];
            out[C + c + i] = ab[j][i];
          }
      } else {
        constexpr int W = LPR * VEC;               // columns of this j
        __syncthreads();
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          s_part[(group * 2) * W + lane * VEC + i] = ag[j][i];
          s_part[(group * 2 + 1) * W + lane * VEC + i] = ab[j][i];
        }
        __syncthreads();
        for (int t = threadIdx.x; t < 2 * W; t += kThreads) {
          float a = 0.0f;
          for (int q = 0; q < G; ++q) a += s_part[q * 2 * W + t];
          const int c = W * j + t % W;
          if (c < C) out[(t / W) * static_cast<int64_t>(C) + c] = a;
        }
      }
    }
  }
}

// Wide rows: dx by a workgroup per row.
template <typename T>
__global__ __launch_bounds__(kThreads) void k_norm_bwd_wide(
    const T* __restrict__ dy, const T* __restrict__ x, const float* __restrict__ mean,
    const float* __restrict__ rstd, const float* __restrict__ gamma, T* __restrict__ dx, int C) {
  constexpr int VEC = Row<T>::VEC;
  __shared__ float s_sum[8];
  const int64_t r = blockIdx.x;
  const float mu = mean[r], rs = rstd[r];
  dy += r * C;
  x += r * C;
  dx += r * C;
  float a = 0.0f, b = 0.0f, ma = 0.0f, mb = 0.0f;
  for (int pass = 0; pass < 2; ++pass) {
    for (int64_t c = threadIdx.x * VEC; c < C; c += kThreads * VEC) {
      float d[VEC], z[VEC], g[VEC];
#pragma unroll
      for (int i = 0; i < VEC; ++i) g[i] = 1.0f;
      if (gamma) load_f32<VEC, true>(gamma, c, C, g);
      load_row<T, true>(dy, c, C, d);
      load_row<T, true>(x, c, C, z);
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        d[i] *= g[i];
        z[i] = c + i < C ? (z[i] - mu) * rs : 0.0f;
        a += d[i];
        b += d[i] * z[i];
        d[i] = rs * (d[i] - ma - z[i] * mb);
      }
      if (pass == 1) store_row<T, true>(dx, c, C, d);
    }
    if (pass == 0) {
      ma = block_sum(a, s_sum, 0) / C;
      mb = block_sum(b, s_sum, 1) / C;
    }
  }
}

// Wide rows: the column sums, a lane per column over the rows of a part.
template <typename T>
__global__ __launch_bounds__(kThreads) void k_norm_cols(
    const T* __restrict__ dy, const T* __restrict__ x, const float* __restrict__ mean,
    const float* __restrict__ rstd, float* __restrict__ part, int64_t n, int C) {
  const int64_t c = static_cast<int64_t>(blockIdx.y) * kThreads + threadIdx.x;
  if (c >= C) return;
  float a = 0.0f, b = 0.0f;
  for (int64_t r = blockIdx.x; r < n; r += gridDim.x) {
    const float d = Row<T>::get(dy[r * C + c]);
    a += d * (Row<T>::get(x[r * C + c]) - mean[r]) * rstd[r];
    b += d;
  }
  float* out = part + static_cast<int64_t>(blockIdx.x) * 2 * C;
  out[c] = a;
  out[C + c] = b;
}

// dgamma | dbeta: the parts' sums, 16 columns by 64 runs of parts per workgroup.
__global__ __launch_bounds__(1024) void k_norm_parts(const float* __restrict__ part, int nparts,
                                                     float* __restrict__ dgamma,
                                                     float* __restrict__ dbeta, int C) {
  __shared__ float s[64][16];
  const int64_t c = static_cast<int64_t>(blockIdx.x) * 16 + (threadIdx.x & 15);
  const int run = threadIdx.x >> 4;
  float a = 0.0f;
  if (c < 2ll * C) {
#pragma unroll 8
    for (int p = run; p < nparts; p += 64) a += part[static_cast<int64_t>(p) * 2 * C + c];
  }
  s[run][threadIdx.x & 15] = a;
  __syncthreads();
  if (run == 0 && c < 2ll * C) {
    a = 0.0f;
    for (int q = 0; q < 64; ++q) a += s[q][threadIdx.x & 15];
    if (c < C) dgamma[c] = a; else dbeta[c - C] = a;
  }
}

// Workgroups of the gradient, each with a part (8 C bytes) of its own: four a
// compute unit, and at least 32 rows each, so that the parts stay a few per cent
// of the rows' own bytes.
int norm_parts(int64_t n) {
  const int64_t p = (n + 31) / 32;
  return static_cast<int>(p < 1 ? 1 : p > 1024 ? 1024 : p);
}

struct NormFwd {
  const void* x;
  const float *gamma, *beta;
  float eps;
  void* y;
  float *mean, *rstd;
  int64_t n;
  int C;
  hipStream_t st;
};
template <typename T, int LPR, int NV, int UR> int run_fwd(const NormFwd& a) {
  constexpr int64_t rows = kThreads / LPR * UR;
  const int64_t blocks = (a.n + rows - 1) / rows;
  if (!grid_fits(blocks, kThreads)) return SPCONV_EINVAL;
  const dim3 grid(static_cast<uint32_t>(blocks));
  const T* x = static_cast<const T*>(a.x);
  T* y = static_cast<T*>(a.y);
  if (a.C % Row<T>::VEC == 0)
    k_norm_fwd<T, LPR, NV, UR, false><<<grid, kThreads, 0, a.st>>>(x, a.gamma, a.beta, a.eps, y,
                                                                  a.mean, a.rstd, a.n, a.C);
  else
    k_norm_fwd<T, LPR, NV, UR, true><<<grid, kThreads, 0, a.st>>>(x, a.gamma, a.beta, a.eps, y,
                                                                 a.mean, a.rstd, a.n, a.C);
  return launched();
}
template <typename T> int norm_fwd(const NormFwd& a) {
  const int64_t pieces = (a.C + Row<T>::VEC - 1) / Row<T>::VEC;
  if (pieces <= 4) return run_fwd<T, 4, 1, 4>(a);
  if (pieces <= 8) return run_fwd<T, 8, 1, 4>(a);
  if (pieces <= 16) return run_fwd<T, 16, 1, 4>(a);
  if (pieces <= 32) return run_fwd<T, 32, 1, 4>(a);
  if (pieces <= 64) return run_fwd<T, 64, 1, 4>(a);
  if (pieces <= 128) return run_fwd<T, 64, 2, 2>(a);
  if (pieces <= 256) return run_fwd<T, 64, 4, 1>(a);
  if (pieces <= 512) return run_fwd<T, 256, 2, 1>(a);
  if (pieces <= 1024) return run_fwd<T, 256, 4, 1>(a);
  if (!grid_fits(a.n, kThreads)) return SPCONV_EINVAL;
  k_norm_fwd_wide<T><<<static_cast<uint32_t>(a.n), kThreads, 0, a.st>>>(
      static_cast<const T*>(a.x), a.gamma, a.beta, a.eps, static_cast<T*>(a.y), a.mean, a.rstd,
      a.C);
  return launched();
}

struct NormBwd {
  const void *dy, *x;
  const float *mean, *rstd, *gamma;
  void* dx;
  float* part;                 // NULL: no parameter gradients
  int nparts;
  int64_t n;
  int C;
  hipStream_t st;
};
template <typename T, int LPR, int NV, int UR> int run_bwd(const NormBwd& a) {
  constexpr int64_t rows = kThreads / LPR * UR;
  const int64_t blocks = (a.n + rows - 1) / rows;
  if (!grid_fits(blocks, kThreads)) return SPCONV_EINVAL;
  const T *dy = static_cast<const T*>(a.dy), *x = static_cast<const T*>(a.x);
  T* dx = static_cast<T*>(a.dx);
  const bool tail = a.C % Row<T>::VEC != 0;
  if (a.part) {
    const dim3 grid(a.nparts);
    if (tail)
      k_norm_bwd<T, LPR, NV, UR, true, true><<<grid, kThreads, 0, a.st>>>(
          dy, x, a.mean, a.rstd, a.gamma, dx, a.part, a.n, a.C);
    else
      k_norm_bwd<T, LPR, NV, UR, false, true><<<grid, kThreads, 0, a.st>>>(
          dy, x, a.mean, a.rstd, a.gamma, dx, a.part, a.n, a.C);
  } else {
    const dim3 grid(static_cast<uint32_t>(blocks));
    if (tail)
      k_norm_bwd<T, LPR, NV, UR, true, false><<<grid, kThreads, 0, a.st>>>(
          dy, x, a.mean, a.rstd, a.gamma, dx, nullptr, a.n, a.C);
    else
      k_norm_bwd<T, LPR, NV, UR, false, false><<<grid, kThreads, 0, a.st>>>(
          dy, x, a.mean, a.rstd, a.gamma, dx, nullptr, a.n, a.C);
  }
  return launched();
}
template <typename T> int norm_bwd(const NormBwd& a) {
  const int64_t pieces = (a.C + Row<T>::VEC - 1) / Row<T>::VEC;
  if (pieces <= 4) return run_bwd<T, 4, 1, 2>(a);
  if (pieces <= 8) return run_bwd<T, 8, 1, 2>(a);
  if (pieces <= 16) return run_bwd<T, 16, 1, 2>(a);
  if (pieces <= 32) return run_bwd<T, 32, 1, 2>(a);
  if (pieces <= 64) return run_bwd<T, 64, 1, 2>(a);
  if (pieces <= 128) return run_bwd<T, 64, 2, 1>(a);
  if (pieces <= 256) return run_bwd<T, 64, 4, 1>(a);
  if (pieces <= 512) return run_bwd<T, 256, 2, 1>(a);
  if (pieces <= 1024) return run_bwd<T, 256, 4, 1>(a);
  const T *dy = static_cast<const T*>(a.dy), *x = static_cast<const T*>(a.x);
  if (!grid_fits(a.n, kThreads)) return SPCONV_EINVAL;
  if (a.n)
    k_norm_bwd_wide<T><<<static_cast<uint32_t>(a.n), kThreads, 0, a.st>>>(
        dy, x, a.mean, a.rstd, a.gamma, static_cast<T*>(a.dx), a.C);
  if (a.part)
    k_norm_cols<T><<<dim3(a.nparts, static_cast<uint32_t>((a.C + kThreads - 1ll) / kThreads)),
                     kThreads, 0, a.st>>>(dy, x, a.mean, a.rstd, a.part, a.n, a.C);
  return launched();
}

bool norm_sizes_ok(int64_t n, int C) { return rows_ok(n) && C >= 1 && C <= 0x7fffff00; }

}  // namespace
}  // namespace spc

using namespace spc;

extern "C" int spconv_layer_norm_forward(int dt, const void* x, const float* gamma,
                                         const float* beta, float eps, void* y, float* mean,
                                         float* rstd, int64_t n, int C, void* stream) {
  if (!dtype_ok(dt) || !norm_sizes_ok(n, C) || !(eps >= 0.0f) || std::isinf(eps) ||
      !ptr_ok(x, n, elem_bytes(dt)) || !ptr_ok(y, n, elem_bytes(dt)) || !aligned_to(gamma, 4) ||
      !aligned_to(beta, 4) || !aligned_to(mean, 4) || !aligned_to(rstd, 4) ||
      (n && !mean != !rstd))
    return SPCONV_EINVAL;
  if (n == 0) return SPCONV_OK;
  const NormFwd a{x, gamma, beta, eps, y, mean, rstd, n, C, static_cast<hipStream_t>(stream)};
  return dt == SPCONV_BF16 ? norm_fwd<bf16_t>(a) : norm_fwd<float>(a);
}

extern "C" int spconv_layer_norm_backward_workspace(int64_t n, int C, size_t* bytes) {
  if (!norm_sizes_ok(n, C) || !bytes) return SPCONV_EINVAL;
  *bytes = static_cast<size_t>(norm_parts(n)) * 2 * C * sizeof(float);
  return SPCONV_OK;
}

extern "C" int spconv_layer_norm_backward(int dt, const void* dy, const void* x, const float* mean,
                                          const float* rstd, const float* gamma, void* dx,
                                          float* dgamma, float* dbeta, int64_t n, int C,
                                          void* workspace, size_t workspace_bytes, void* stream) {
  if (!dtype_ok(dt) || !norm_sizes_ok(n, C) || !dgamma != !dbeta || !aligned_to(dgamma, 4) ||
      !aligned_to(dbeta, 4) || !aligned_to(gamma, 4))
    return SPCONV_EINVAL;
  const size_t e = elem_bytes(dt);
  if (!ptr_ok(dy, n, e) || !ptr_ok(x, n, e) || !ptr_ok(dx, n, e) || !ptr_ok(mean, n, 4) ||
      !ptr_ok(rstd, n, 4))
    return SPCONV_EINVAL;
  const int nparts = norm_parts(n);
  // k_norm_cols: a column of workgroups per part, at most 65,535 rows of them
  if (dgamma && (C > 65535 * kThreads || !grid_fits(nparts * (C / kThreads + 1ll), kThreads)))
    return SPCONV_EINVAL;
  if (dgamma && (!workspace || !aligned_to(workspace, 16) ||
                 workspace_bytes < static_cast<size_t>(nparts) * 2 * C * sizeof(float)))
    return SPCONV_EINVAL;
  if (n == 0 && !dgamma) return SPCONV_OK;
  hipStream_t st = static_cast<hipStream_t>(stream);
  float* part = dgamma ? static_cast<float*>(workspace) : nullptr;
  const NormBwd a{dy, x, mean, rstd, gamma, dx, part, nparts, n, C, st};
  const int status = dt == SPCONV_BF16 ? norm_bwd<bf16_t>(a) : norm_bwd<float>(a);
  if (status != SPCONV_OK) return status;
  if (dgamma)
    k_norm_parts<<<static_cast<uint32_t>((2ll * C + 15) / 16), 1024, 0, st>>>(part, nparts, dgamma,
                                                                            dbeta, C);
  return launched();
}
