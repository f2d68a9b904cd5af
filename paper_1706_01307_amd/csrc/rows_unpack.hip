// Rows in 8 bits as values again, through an activation, and the gradient of an activation
// whose input is at hand in either form.
//
// Elementwise and bound by memory.  A group of lanes takes a row at a time, so that its
// scale is one load and no element asks which row it is in; as many lanes as a row has
// pieces, to a power of two (348,208 bf16 rows of 256, half of the lanes idle: 81 us for the
// GELU of them, 42 so, 6.3 TB/s; its derivative times dy 140, and 80, 5.6).
#include "rows_act.h"

namespace spc {
namespace {

constexpr int kThreads = 256;

struct ActArgs {
  const void *dy, *z;          // dy NULL: the activation itself
  const float* scale;
  void* out;
  int64_t n;
  int C;
  hipStream_t st;
};

// Z8: z in 8 bits.  GRAD: out = dy * slope(z), else activate(z).  LPR lanes a row, UR rows of
// a group and a piece of each at a time; wider rows in turns.
template <typename T, bool Z8, bool GRAD, int ACT, int LPR, bool TAIL>
__global__ __launch_bounds__(kThreads) void k_act(ActArgs a) {
  constexpr int VEC = Row<T>::VEC, G = kThreads / LPR, UR = 4;
  const T *const dy = static_cast<const T*>(a.dy), *const z = static_cast<const T*>(a.z);
  T* const out = static_cast<T*>(a.out);
  const int C = a.C;
  const int64_t first = (static_cast<int64_t>(blockIdx.x) * G + threadIdx.x / LPR) * UR;
  float s[UR];
#pragma unroll
  for (int u = 0; u < UR; ++u) s[u] = Z8 && first + u < a.n ? a.scale[first + u] : 1.0f;
  for (int64_t c = static_cast<int64_t>(threadIdx.x % LPR) * VEC; c < C; c += LPR * VEC) {
    float v[UR][VEC], d[UR][VEC];
#pragma unroll
    for (int u = 0; u < UR; ++u) {
      if (first + u >= a.n) break;
      const int64_t r = (first + u) * C;
      if constexpr (Z8) load_row8<VEC, TAIL>(static_cast<const uint8_t*>(a.z) + r, c, C, v[u]);
      else load_row<T, TAIL>(z + r, c, C, v[u]);
      if constexpr (GRAD) load_row<T, TAIL>(dy + r, c, C, d[u]);
    }
#pragma unroll
    for (int u = 0; u < UR; ++u) {
      if (first + u >= a.n) break;
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        const float w = Z8 ? v[u][i] * s[u] : v[u][i];
        v[u][i] = GRAD ? d[u][i] * slope<ACT, sizeof(T) == 4>(w)
                       : activate<ACT, sizeof(T) == 4>(w);
      }
      store_row<T, TAIL>(out + (first + u) * C, c, C, v[u]);
    }
  }
}

template <typename T, bool Z8, bool GRAD, int ACT, int LPR> int run_lanes(const ActArgs& a) {
  constexpr int64_t rows = kThreads / LPR * 4;
  const int64_t blocks = (a.n + rows - 1) / rows;
  if (!grid_fits(blocks, kThreads)) return SPCONV_EINVAL;
  const uint32_t grid = static_cast<uint32_t>(blocks);
  if (a.C % Row<T>::VEC) k_act<T, Z8, GRAD, ACT, LPR, true><<<grid, kThreads, 0, a.st>>>(a);
  else k_act<T, Z8, GRAD, ACT, LPR, false><<<grid, kThreads, 0, a.st>>>(a);
  return launched();
}
template <typename T, bool Z8, bool GRAD> int run(int act, const ActArgs& a) {
  const int64_t pieces = (a.C + Row<T>::VEC - 1) / Row<T>::VEC;
  return by_act(act, [&](auto k) {
    constexpr int ACT = decltype(k)::value;
    if (pieces <= 4) return run_lanes<T, Z8, GRAD, ACT, 4>(a);
    if (pieces <= 8) return run_lanes<T, Z8, GRAD, ACT, 8>(a);
    if (pieces <= 16) return run_lanes<T, Z8, GRAD, ACT, 16>(a);
    if (pieces <= 32) return run_lanes<T, Z8, GRAD, ACT, 32>(a);
    return run_lanes<T, Z8, GRAD, ACT, 64>(a);
  });
}

bool act_sizes_ok(int64_t n, int C) { return rows_ok(n) && C >= 1 && C <= 0x7fffff00; }

}  // namespace
}  // namespace spc

using namespace spc;

extern "C" int spconv_unpack_rows(const void* q, const float* scale, int act, int out_dt, void* y,
                                  int64_t n, int C, void* stream) {
  if (!dtype_ok(out_dt) || !act_ok(act) || !act_sizes_ok(n, C) || !ptr_ok(q, n, 1) ||
      !ptr_ok(scale, n, 4) || !ptr_ok(y, n, elem_bytes(out_dt)))
    return SPCONV_EINVAL;
  if (n == 0) return SPCONV_OK;
  const ActArgs a{nullptr, q, scale, y, n, C, static_cast<hipStream_t>(stream)};
  return out_dt == SPCONV_BF16 ? run<bf16_t, true, false>(act, a) : run<float, true, false>(act, a);
}

extern "C" int spconv_activation_backward(int dt, const void* dy, int pre_dt, const void* pre,
                                          const float* pre_scale, int act, void* dz, int64_t n,
                                          int C, void* stream) {
  if (!dtype_ok(dt) || (pre_dt != dt && pre_dt != SPCONV_E4M3) || !act_ok(act) ||
      !act_sizes_ok(n, C))
    return SPCONV_EINVAL;
  const size_t e = elem_bytes(dt);
  const bool e4m3 = pre_dt == SPCONV_E4M3;
  if (!ptr_ok(dy, n, e) || !ptr_ok(pre, n, e4m3 ? 1 : e) || !ptr_ok(pre_scale, e4m3 ? n : 0, 4) ||
      (pre_scale && !e4m3) || !ptr_ok(dz, n, e))
    return SPCONV_EINVAL;
  if (n == 0) return SPCONV_OK;
  const ActArgs a{dy, pre, pre_scale, dz, n, C, static_cast<hipStream_t>(stream)};
  if (dt == SPCONV_BF16)
    return e4m3 ? run<bf16_t, true, true>(act, a) : run<bf16_t, false, true>(act, a);
  return e4m3 ? run<float, true, true>(act, a) : run<float, false, true>(act, a);
}
