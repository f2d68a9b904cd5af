// Root-mean-square norm of feature rows with the residual's addition, its output in the
// rows' type or in 8 bits, and its gradients; rows packed into 8 bits.
//
// One pass over the rows, as for layer norm: a row lives in the registers of a group of
// lanes between its statistics (sum of squares, then largest magnitude) and its outputs, so
// that memory is read and written once; the group's sums go over the vector ALU's lane
// permutations.  Bound by memory bandwidth (a large copy reaches 5.1 TB/s): 902,504 bf16 rows
// of 64 with a residual take 82 us forwards (5.6 TB/s) and 97 + 5 backwards (4.8), 348,208 of
// 256 to 8 bits 115 (5.4), packed alone 44 (6.1); 87,052 fp32 rows of 145 backwards from 8
// bits 37 + 4 us (4.5).
#include <cmath>

#include "rows_act.h"

namespace spc {
namespace {

constexpr int kThreads = 256;

// Sums and largest magnitudes over the LPR lanes that hold a row (256: the workgroup).
template <int LPR> struct RowReduce {
  float* s;
  int turn = 0;
  __device__ explicit RowReduce(float* lds) : s(lds) {}
  __device__ float sum(float v) {
    if constexpr (LPR <= 64) return group_sum<LPR>(v);
    return block_sum(v, s, turn++);
  }
  __device__ float top(float v) {
    v = group_reduce<LPR <= 64 ? LPR : 64>(v, larger_magnitude);
    if constexpr (LPR > 64) {
      float* t = s + 4 * (turn++ & 1);
      if ((threadIdx.x & 63) == 0) t[threadIdx.x >> 6] = v;
      __syncthreads();
      v = larger_magnitude(larger_magnitude(t[0], t[1]), larger_magnitude(t[2], t[3]));
    }
    return v;
  }
};

struct RmsFwd {
  const void *x, *res;
  const float* gamma;
  float eps;
  void *h, *y;
  float *scale, *rstd;
  int64_t n;
  int C;
  hipStream_t st;
};

// h = x + res rounded to the rows' type, rstd = 1 / sqrt(mean of h^2 + eps), y = h rstd gamma.
// (The statistics are those of h as it is stored, so that the gradient, which reads it, is
// the gradient of what was computed.)  E4M3: y goes to 8 bits straight from fp32.  NORM false:
// no norm, the rows themselves are packed.  A group of LPR lanes holds a row of at most LPR *
// NV * VEC elements and takes UR rows at a time, their loads in flight together.
template <typename T, bool NORM, bool E4M3, int LPR, int NV, int UR, bool TAIL>
__global__ __launch_bounds__(kThreads) void k_rms_fwd(RmsFwd a) {
  constexpr int VEC = Row<T>::VEC, G = kThreads / LPR;
  __shared__ float s_red[8];
  RowReduce<LPR> over(s_red);
  const T *const x = static_cast<const T*>(a.x), *const res = static_cast<const T*>(a.res);
  T* const h = static_cast<T*>(a.h);
  const int C = a.C, lane = threadIdx.x % LPR;
  const int64_t first = (static_cast<int64_t>(blockIdx.x) * G + threadIdx.x / LPR) * UR;
  float v[UR][NV][VEC];
#pragma unroll
  for (int u = 0; u < UR; ++u)
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (lane + LPR * j) * VEC;
#pragma unroll
      for (int i = 0; i < VEC; ++i) v[u][j][i] = 0.0f;
      if (first + u < a.n && c < C) load_row<T, TAIL>(x + (first + u) * C, c, C, v[u][j]);
    }
  if (NORM && res) {
    float w[UR][NV][VEC];
#pragma unroll
    for (int u = 0; u < UR; ++u)
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const int c = (lane + LPR * j) * VEC;
#pragma unroll
        for (int i = 0; i < VEC; ++i) w[u][j][i] = 0.0f;
        if (first + u < a.n && c < C) load_row<T, TAIL>(res + (first + u) * C, c, C, w[u][j]);
      }
#pragma unroll
    for (int u = 0; u < UR; ++u)
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const int c = (lane + LPR * j) * VEC;
#pragma unroll
        for (int i = 0; i < VEC; ++i) v[u][j][i] = Row<T>::get(Row<T>::put(v[u][j][i] + w[u][j][i]));
        if (h && first + u < a.n && c < C) store_row<T, TAIL>(h + (first + u) * C, c, C, v[u][j]);
      }
  }
  float rs[UR];
  if constexpr (NORM) {
#pragma unroll
    for (int u = 0; u < UR; ++u) {
      float s = 0.0f;
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < VEC; ++i) s += v[u][j][i] * v[u][j][i];
      rs[u] = 1.0f / sqrtf(over.sum(s) / C + a.eps);
    }
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (lane + LPR * j) * VEC;
      float g[VEC];
#pragma unroll
      for (int i = 0; i < VEC; ++i) g[i] = 1.0f;
      if (a.gamma && c < C) load_f32<VEC, TAIL>(a.gamma, c, C, g);
#pragma unroll
      for (int u = 0; u < UR; ++u) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) v[u][j][i] = v[u][j][i] * rs[u] * g[i];
        if (!E4M3 && first + u < a.n && c < C)
          store_row<T, TAIL>(static_cast<T*>(a.y) + (first + u) * C, c, C, v[u][j]);
      }
    }
    if (a.rstd && lane == 0)
#pragma unroll
      for (int u = 0; u < UR; ++u)
        if (first + u < a.n) a.rstd[first + u] = rs[u];
  }
  if constexpr (E4M3) {
#pragma unroll
    for (int u = 0; u < UR; ++u) {
      float top = 0.0f, scale, inverse;
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < VEC; ++i)
          top = larger_magnitude(top, __uint_as_float(magnitude(v[u][j][i])));
      scale_of(over.top(top), &scale, &inverse);
      if (first + u >= a.n) continue;
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const int c = (lane + LPR * j) * VEC;
        if (c < C)
          store_row8<VEC, TAIL>(static_cast<uint8_t*>(a.y) + (first + u) * C, c, C, v[u][j],
                                inverse);
      }
      if (lane == 0) a.scale[first + u] = scale;
    }
  }
}

// Rows too wide for a workgroup's registers: a workgroup per row, which it reads two or
// three times (from the caches after the first).
template <typename T, bool NORM, bool E4M3>
__global__ __launch_bounds__(kThreads) void k_rms_fwd_wide(RmsFwd a) {
  constexpr int VEC = Row<T>::VEC;
  __shared__ float s_red[8];
  RowReduce<kThreads> over(s_red);
  const int64_t r = blockIdx.x, C = a.C, step = kThreads * VEC, c0 = threadIdx.x * VEC;
  const T* x = static_cast<const T*>(a.x) + r * C;
  const T* const res = NORM && a.res ? static_cast<const T*>(a.res) + r * C : nullptr;
  T* const h = a.h ? static_cast<T*>(a.h) + r * C : nullptr;
  float v[VEC];
  auto load = [&](int64_t c) {
    load_row<T, true>(x, c, C, v);
    if (!res) return;
    float w[VEC];
    load_row<T, true>(res, c, C, w);
#pragma unroll
    for (int i = 0; i < VEC; ++i) v[i] = Row<T>::get(Row<T>::put(v[i] + w[i]));
  };
  float rs = 1.0f, s = 0.0f;
  if constexpr (NORM) {
    for (int64_t c = c0; c < C; c += step) {
      load(c);
#pragma unroll
      for (int i = 0; i < VEC; ++i) s += v[i] * v[i];
    }
    rs = 1.0f / sqrtf(over.sum(s) / C + a.eps);
    if (a.rstd && threadIdx.x == 0) a.rstd[r] = rs;
  }
  auto normed = [&](int64_t c) {
    if constexpr (NORM) {
      float g[VEC];
#pragma unroll
      for (int i = 0; i < VEC; ++i) g[i] = 1.0f;
      if (a.gamma) load_f32<VEC, true>(a.gamma, c, C, g);
#pragma unroll
      for (int i = 0; i < VEC; ++i) v[i] = v[i] * rs * g[i];
    }
  };
  float scale, inverse = 1.0f;
  if constexpr (E4M3) {
    float top = 0.0f;
    for (int64_t c = c0; c < C; c += step) {
      load(c);
      normed(c);
#pragma unroll
      for (int i = 0; i < VEC; ++i) top = larger_magnitude(top, __uint_as_float(magnitude(v[i])));
    }
    scale_of(over.top(top), &scale, &inverse);
    if (threadIdx.x == 0) a.scale[r] = scale;
  }
  // (h may be x or res itself: nobody else reads these elements, and this is the last time)
  for (int64_t c = c0; c < C; c += step) {
    load(c);
    if (res && h) store_row<T, true>(h, c, C, v);
    normed(c);
    if constexpr (E4M3)
      store_row8<VEC, true>(static_cast<uint8_t*>(a.y) + r * C, c, C, v, inverse);
    else
      store_row<T, true>(static_cast<T*>(a.y) + r * C, c, C, v);
  }
}

struct RmsBwd {
  const void *dy, *h;
  const float *h_scale, *rstd, *gamma;
  const void* dh;
  void* dx;
  float* part;                 // NULL: no gradient of gamma
  int nparts;
  int64_t n;
  int C;
  hipStream_t st;
};

// The sum as the gradient reads it: of the rows' type, or (H8) in 8 bits without its scale.
template <typename T, bool H8, bool TAIL>
__device__ __forceinline__ void load_sum(const void* h, int64_t r, int64_t c, int64_t C,
                                         float (&v)[Row<T>::VEC]) {
  if constexpr (H8) load_row8<Row<T>::VEC, TAIL>(static_cast<const uint8_t*>(h) + r * C, c, C, v);
  else load_row<T, TAIL>(static_cast<const T*>(h) + r * C, c, C, v);
}

// With z = h rstd and d = gamma dy: dx = rstd (d - z mean of d z) + dh.  With PARAM, a lane
// keeps its columns' sums of dy z over the rows its group takes (every gridDim.x * G-th batch
// of UR rows); the groups' sums are added through LDS in group order and leave as the
// workgroup's row of `part`, which k_rms_parts adds up.
template <typename T, bool H8, int LPR, int NV, int UR, bool TAIL, bool PARAM>
__global__ __launch_bounds__(kThreads) void k_rms_bwd(RmsBwd a) {
  constexpr int VEC = Row<T>::VEC, G = kThreads / LPR;
  __shared__ float s_red[8];
  RowReduce<LPR> over(s_red);
  const T *const dy = static_cast<const T*>(a.dy), *const dh = static_cast<const T*>(a.dh);
  T* const dx = static_cast<T*>(a.dx);
  const int C = a.C, lane = threadIdx.x % LPR, group = threadIdx.x / LPR;
  float g[NV][VEC], ag[PARAM ? NV : 1][VEC];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int c = (lane + LPR * j) * VEC;
#pragma unroll
    for (int i = 0; i < VEC; ++i) g[j][i] = 1.0f;
    if (a.gamma && c < C) load_f32<VEC, TAIL>(a.gamma, c, C, g[j]);
    if constexpr (PARAM) {
#pragma unroll
      for (int i = 0; i < VEC; ++i) ag[j][i] = 0.0f;
    }
  }
  const int64_t stride = static_cast<int64_t>(gridDim.x) * G * UR;
  // uniform over the workgroup (the sums have barriers)
  for (int64_t base = static_cast<int64_t>(blockIdx.x) * G * UR; base < a.n; base += stride) {
    const int64_t first = base + static_cast<int64_t>(group) * UR;
    float d[UR][NV][VEC], z[UR][NV][VEC], e[UR][NV][VEC], rs[UR], zs[UR];
#pragma unroll
    for (int u = 0; u < UR; ++u) {
      const bool live = first + u < a.n;
      rs[u] = live ? a.rstd[first + u] : 0.0f;
      zs[u] = rs[u];
      if (H8 && live) zs[u] *= a.h_scale[first + u];
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const int c = (lane + LPR * j) * VEC;
#pragma unroll
        for (int i = 0; i < VEC; ++i) d[u][j][i] = z[u][j][i] = e[u][j][i] = 0.0f;
        if (live && c < C) {
          load_row<T, TAIL>(dy + (first + u) * C, c, C, d[u][j]);
          load_sum<T, H8, TAIL>(a.h, first + u, c, C, z[u][j]);
          if (dh) load_row<T, TAIL>(dh + (first + u) * C, c, C, e[u][j]);
        }
      }
    }
#pragma unroll
    for (int u = 0; u < UR; ++u) {
      float s = 0.0f;
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          z[u][j][i] *= zs[u];
          if constexpr (PARAM) ag[j][i] += d[u][j][i] * z[u][j][i];
          d[u][j][i] *= g[j][i];
          s += d[u][j][i] * z[u][j][i];
        }
      const float mean = over.sum(s) / C;
      if (first + u < a.n) {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
          const int c = (lane + LPR * j) * VEC;
          if (c >= C) continue;
          float o[VEC];
#pragma unroll
          for (int i = 0; i < VEC; ++i) o[i] = rs[u] * (d[u][j][i] - z[u][j][i] * mean) + e[u][j][i];
          store_row<T, TAIL>(dx + (first + u) * C, c, C, o);
        }
      }
    }
  }
  if constexpr (PARAM) {
    float* out = a.part + static_cast<int64_t>(blockIdx.x) * C;
    __shared__ float s_part[G > 1 ? kThreads * VEC : 1];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      if constexpr (G == 1) {
        const int c = (lane + LPR * j) * VEC;
#pragma unroll
        for (int i = 0; i < VEC; ++i)
          if (c + i < C) out[c + i] = ag[j][i];
      } else {
        constexpr int W = LPR * VEC;               // columns of this j
        __syncthreads();
#pragma unroll
        for (int i = 0; i < VEC; ++i) s_part[group * W + lane * VEC + i] = ag[j][i];
        __syncthreads();
        for (int t = threadIdx.x; t < W; t += kThreads) {
          float s = 0.0f;
          for (int q = 0; q < G; ++q) s += s_part[q * W + t];
          if (W * j + t < C) out[W * j + t] = s;
        }
      }
    }
  }
}

// Wide rows: dx by a workgroup per row.
template <typename T, bool H8>
__global__ __launch_bounds__(kThreads) void k_rms_bwd_wide(RmsBwd a) {
  constexpr int VEC = Row<T>::VEC;
  __shared__ float s_red[8];
  const int64_t r = blockIdx.x, C = a.C;
  const T* const dy = static_cast<const T*>(a.dy) + r * C;
  const T* const dh = a.dh ? static_cast<const T*>(a.dh) + r * C : nullptr;
  const float rs = a.rstd[r], zs = H8 ? rs * a.h_scale[r] : rs;
  float s = 0.0f, mean = 0.0f;
  for (int pass = 0; pass < 2; ++pass) {
    for (int64_t c = threadIdx.x * VEC; c < C; c += kThreads * VEC) {
      float d[VEC], z[VEC], g[VEC], e[VEC];
#pragma unroll
      for (int i = 0; i < VEC; ++i) g[i] = 1.0f, e[i] = 0.0f;
      if (a.gamma) load_f32<VEC, true>(a.gamma, c, C, g);
      load_row<T, true>(dy, c, C, d);
      load_sum<T, H8, true>(a.h, r, c, C, z);
      if (pass && dh) load_row<T, true>(dh, c, C, e);
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        d[i] *= g[i];
        z[i] *= zs;
        s += d[i] * z[i];
        d[i] = rs * (d[i] - z[i] * mean) + e[i];
      }
      if (pass) store_row<T, true>(static_cast<T*>(a.dx) + r * C, c, C, d);
    }
    if (!pass) mean = block_sum(s, s_red, 0) / C;
  }
}

// Wide rows: the column sums, a lane per column over the rows of a part.
template <typename T, bool H8>
__global__ __launch_bounds__(kThreads) void k_rms_cols(RmsBwd a) {
  const int64_t C = a.C, c = static_cast<int64_t>(blockIdx.y) * kThreads + threadIdx.x;
  if (c >= C) return;
  float s = 0.0f;
  for (int64_t r = blockIdx.x; r < a.n; r += gridDim.x) {
    float z;
    if constexpr (H8) {
      const uint32_t q = static_cast<const uint8_t*>(a.h)[r * C + c];
      z = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(q), false)[0] * a.h_scale[r];
    } else {
      z = Row<T>::get(static_cast<const T*>(a.h)[r * C + c]);
    }
    s += Row<T>::get(static_cast<const T*>(a.dy)[r * C + c]) * z * a.rstd[r];
  }
  a.part[static_cast<int64_t>(blockIdx.x) * C + c] = s;
}

// dgamma: the parts' sums, 16 columns by 64 runs of parts per workgroup.
__global__ __launch_bounds__(1024) void k_rms_parts(const float* __restrict__ part, int nparts,
                                                    float* __restrict__ dgamma, int C) {
  __shared__ float s[64][16];
  const int64_t c = static_cast<int64_t>(blockIdx.x) * 16 + (threadIdx.x & 15);
  const int run = threadIdx.x >> 4;
  float a = 0.0f;
  if (c < C) {
#pragma unroll 8
    for (int p = run; p < nparts; p += 64) a += part[static_cast<int64_t>(p) * C + c];
  }
  s[run][threadIdx.x & 15] = a;
  __syncthreads();
  if (run == 0 && c < C) {
    a = 0.0f;
    for (int q = 0; q < 64; ++q) a += s[q][threadIdx.x & 15];
    dgamma[c] = a;
  }
}

// Workgroups of the gradient, each with a part (4 C bytes) of its own: four a compute
// unit, and at least 32 rows each, so that the parts stay a few per cent of the rows' own
// bytes.
int rms_parts(int64_t n) {
  const int64_t p = (n + 31) / 32;
  return static_cast<int>(p < 1 ? 1 : p > 1024 ? 1024 : p);
}

template <bool NORM, bool E4M3, typename T, int LPR, int NV, int UR> int run(const RmsFwd& a) {
  constexpr int64_t rows = kThreads / LPR * UR;
  const int64_t blocks = (a.n + rows - 1) / rows;
  if (!grid_fits(blocks, kThreads)) return SPCONV_EINVAL;
  const dim3 grid(static_cast<uint32_t>(blocks));
  if (a.C % Row<T>::VEC == 0)
    k_rms_fwd<T, NORM, E4M3, LPR, NV, UR, false><<<grid, kThreads, 0, a.st>>>(a);
  else
    k_rms_fwd<T, NORM, E4M3, LPR, NV, UR, true><<<grid, kThreads, 0, a.st>>>(a);
  return launched();
}
template <bool NORM, bool E4M3, typename T> int rms_fwd(const RmsFwd& a) {
  const int64_t pieces = (a.C + Row<T>::VEC - 1) / Row<T>::VEC;
  if (pieces <= 4) return run<NORM, E4M3, T, 4, 1, 4>(a);
  if (pieces <= 8) return run<NORM, E4M3, T, 8, 1, 4>(a);
  if (pieces <= 16) return run<NORM, E4M3, T, 16, 1, 4>(a);
  if (pieces <= 32) return run<NORM, E4M3, T, 32, 1, 4>(a);
  if (pieces <= 64) return run<NORM, E4M3, T, 64, 1, 4>(a);
  if (pieces <= 128) return run<NORM, E4M3, T, 64, 2, 2>(a);
  if (pieces <= 256) return run<NORM, E4M3, T, 64, 4, 1>(a);
  if (pieces <= 512) return run<NORM, E4M3, T, 256, 2, 1>(a);
  if (pieces <= 1024) return run<NORM, E4M3, T, 256, 4, 1>(a);
  if (!grid_fits(a.n, kThreads)) return SPCONV_EINVAL;
  k_rms_fwd_wide<T, NORM, E4M3><<<static_cast<uint32_t>(a.n), kThreads, 0, a.st>>>(a);
  return launched();
}

template <bool H8, typename T, int LPR, int NV, int UR> int run(const RmsBwd& a) {
  constexpr int64_t rows = kThreads / LPR * UR;
  const int64_t blocks = (a.n + rows - 1) / rows;
  if (!grid_fits(blocks, kThreads)) return SPCONV_EINVAL;
  const bool tail = a.C % Row<T>::VEC != 0;
  if (a.part) {
    if (tail) k_rms_bwd<T, H8, LPR, NV, UR, true, true><<<a.nparts, kThreads, 0, a.st>>>(a);
    else k_rms_bwd<T, H8, LPR, NV, UR, false, true><<<a.nparts, kThreads, 0, a.st>>>(a);
  } else {
    const uint32_t grid = static_cast<uint32_t>(blocks);
    if (tail) k_rms_bwd<T, H8, LPR, NV, UR, true, false><<<grid, kThreads, 0, a.st>>>(a);
    else k_rms_bwd<T, H8, LPR, NV, UR, false, false><<<grid, kThreads, 0, a.st>>>(a);
  }
  return launched();
}
template <bool H8, typename T> int rms_bwd(const RmsBwd& a) {
  const int64_t pieces = (a.C + Row<T>::VEC - 1) / Row<T>::VEC;
  if (pieces <= 4) return run<H8, T, 4, 1, 2>(a);
  if (pieces <= 8) return run<H8, T, 8, 1, 2>(a);
  if (pieces <= 16) return run<H8, T, 16, 1, 2>(a);
  if (pieces <= 32) return run<H8, T, 32, 1, 2>(a);
  if (pieces <= 64) return run<H8, T, 64, 1, 2>(a);
  if (pieces <= 128) return run<H8, T, 64, 2, 1>(a);
  if (pieces <= 256) return run<H8, T, 64, 4, 1>(a);
  if (pieces <= 512) return run<H8, T, 256, 2, 1>(a);
  if (pieces <= 1024) return run<H8, T, 256, 4, 1>(a);
  if (!grid_fits(a.n, kThreads)) return SPCONV_EINVAL;
  if (a.n) k_rms_bwd_wide<T, H8><<<static_cast<uint32_t>(a.n), kThreads, 0, a.st>>>(a);
  if (a.part)
    k_rms_cols<T, H8><<<dim3(a.nparts, static_cast<uint32_t>((a.C + kThreads - 1ll) / kThreads)),
                        kThreads, 0, a.st>>>(a);
  return launched();
}

bool rms_sizes_ok(int64_t n, int C) { return rows_ok(n) && C >= 1 && C <= 0x7fffff00; }

}  // namespace
}  // namespace spc

using namespace spc;

extern "C" int spconv_rms_norm_forward(int dt, const void* x, const void* residual,
                                       const float* gamma, float eps, void* h, int out_dt, void* y,
                                       float* y_scale, float* rstd, int64_t n, int C,
                                       void* stream) {
  if (!dtype_ok(dt) || (out_dt != dt && out_dt != SPCONV_E4M3) || !rms_sizes_ok(n, C) ||
      !(eps >= 0.0f) || std::isinf(eps))
    return SPCONV_EINVAL;
  const size_t e = elem_bytes(dt);
  const bool e4m3 = out_dt == SPCONV_E4M3;
  if (!ptr_ok(x, n, e) || !aligned_to(residual, e) || !aligned_to(gamma, 4) || !aligned_to(h, e) ||
      (h && !residual) || !ptr_ok(y, n, e4m3 ? 1 : e) || !ptr_ok(y_scale, e4m3 ? n : 0, 4) ||
      (y_scale && !e4m3) || !aligned_to(rstd, 4))
    return SPCONV_EINVAL;
  if (n == 0) return SPCONV_OK;
  const RmsFwd a{x, residual, gamma, eps, h, y, y_scale, rstd, n, C,
                 static_cast<hipStream_t>(stream)};
  if (dt == SPCONV_BF16) return e4m3 ? rms_fwd<true, true, bf16_t>(a) : rms_fwd<true, false, bf16_t>(a);
  return e4m3 ? rms_fwd<true, true, float>(a) : rms_fwd<true, false, float>(a);
}

extern "C" int spconv_rms_norm_backward_workspace(int64_t n, int C, size_t* bytes) {
  if (!rms_sizes_ok(n, C) || !bytes) return SPCONV_EINVAL;
  *bytes = static_cast<size_t>(rms_parts(n)) * C * sizeof(float);
  return SPCONV_OK;
}

extern "C" int spconv_rms_norm_backward(int dt, const void* dy, int h_dt, const void* h,
                                        const float* h_scale, const float* rstd,
                                        const float* gamma, const void* dh, void* dx,
                                        float* dgamma, int64_t n, int C, void* workspace,
                                        size_t workspace_bytes, void* stream) {
  if (!dtype_ok(dt) || (h_dt != dt && h_dt != SPCONV_E4M3) || !rms_sizes_ok(n, C))
    return SPCONV_EINVAL;
  const size_t e = elem_bytes(dt);
  const bool e4m3 = h_dt == SPCONV_E4M3;
  if (!ptr_ok(dy, n, e) || !ptr_ok(h, n, e4m3 ? 1 : e) || !ptr_ok(h_scale, e4m3 ? n : 0, 4) ||
      (h_scale && !e4m3) || !ptr_ok(rstd, n, 4) || !aligned_to(gamma, 4) || !aligned_to(dh, e) ||
      !ptr_ok(dx, n, e) || !aligned_to(dgamma, 4))
    return SPCONV_EINVAL;
  const int nparts = rms_parts(n);
  // k_rms_cols: a column of workgroups per part, at most 65,535 rows of them
  if (dgamma && (C > 65535 * kThreads || !grid_fits(nparts * (C / kThreads + 1ll), kThreads)))
    return SPCONV_EINVAL;
  if (dgamma && (!workspace || !aligned_to(workspace, 16) ||
                 workspace_bytes < static_cast<size_t>(nparts) * C * sizeof(float)))
    return SPCONV_EINVAL;
  if (n == 0 && !dgamma) return SPCONV_OK;
  hipStream_t st = static_cast<hipStream_t>(stream);
  float* part = dgamma ? static_cast<float*>(workspace) : nullptr;
  const RmsBwd a{dy, h, h_scale, rstd, gamma, dh, dx, part, nparts, n, C, st};
  const int status = dt == SPCONV_BF16
                         ? (e4m3 ? rms_bwd<true, bf16_t>(a) : rms_bwd<false, bf16_t>(a))
                         : (e4m3 ? rms_bwd<true, float>(a) : rms_bwd<false, float>(a));
  if (status != SPCONV_OK) return status;
  if (dgamma)
    k_rms_parts<<<static_cast<uint32_t>((C + 15ll) / 16), 1024, 0, st>>>(part, nparts, dgamma, C);
  return launched();
}

extern "C" int spconv_pack_rows(int dt, const void* x, void* q, float* scale, int64_t n, int C,
                                void* stream) {
  if (!dtype_ok(dt) || !rms_sizes_ok(n, C) || !ptr_ok(x, n, elem_bytes(dt)) || !ptr_ok(q, n, 1) ||
      !ptr_ok(scale, n, 4))
    return SPCONV_EINVAL;
  if (n == 0) return SPCONV_OK;
  const RmsFwd a{x, nullptr, nullptr, 0.0f, nullptr, q, scale, nullptr, n, C,
                 static_cast<hipStream_t>(stream)};
  return dt == SPCONV_BF16 ? rms_fwd<false, true, bf16_t>(a) : rms_fwd<false, true, float>(a);
}
