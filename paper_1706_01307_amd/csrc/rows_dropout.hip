// Dropout from a counter-based generator: the same map of elements forwards and
// backwards, recomputed from (seed, offset, element index), never stored.
//
// Philox4x32 (Salmon, Moraes, Dror and Shaw, 2011) makes four 32-bit words of a
// counter by rounds of two 32 x 32 -> 64 bit products.  Seven rounds are the
// fewest its authors found to pass their whole battery of tests.
#include <cmath>
#include <type_traits>

#include "rows.h"

namespace spc {
namespace {

constexpr int kThreads = 256;
constexpr int kRounds = 7;

__device__ __forceinline__ void philox(uint64_t index, uint64_t offset, uint64_t seed,
                                       uint32_t (&w)[4]) {
  uint32_t c0 = static_cast<uint32_t>(index), c1 = static_cast<uint32_t>(index >> 32);
  uint32_t c2 = static_cast<uint32_t>(offset), c3 = static_cast<uint32_t>(offset >> 32);
  uint32_t k0 = static_cast<uint32_t>(seed), k1 = static_cast<uint32_t>(seed >> 32);
#pragma unroll
  for (int r = 0; r < kRounds; ++r) {
    const uint64_t a = static_cast<uint64_t>(c0) * 0xD2511F53u;
    const uint64_t b = static_cast<uint64_t>(c2) * 0xCD9E8D57u;
    c0 = static_cast<uint32_t>(b >> 32) ^ c1 ^ k0;
    c1 = static_cast<uint32_t>(b);
    c2 = static_cast<uint32_t>(a >> 32) ^ c3 ^ k1;
    c3 = static_cast<uint32_t>(a);
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  w[0] = c0; w[1] = c1; w[2] = c2; w[3] = c3;
}

// y = res + (word >= threshold ? x / (1 - p) : 0), added in fp32 and rounded once.
// Bound by memory bandwidth: 902,504 x 64 bf16 with a residual take 64 us, 5.4 TB/s
// (a large copy reaches 5.1); the products of the generator hide behind the loads.
// A lane takes one 16-byte piece (4 or 8 elements: one or two counters) of each
// of NP strips, their loads in flight together.  x and y may be the same, as
// may res and y: a lane reads what it overwrites, first.
template <typename T, bool RES, int NP>
__global__ __launch_bounds__(kThreads) void k_dropout(const T* x, const T* res, uint64_t threshold,
                                                      float scale, uint64_t seed, uint64_t offset,
                                                      const uint64_t* __restrict__ step, T* y,
                                                      int64_t count) {
  constexpr int VEC = Row<T>::VEC;
  if (step) offset += *step;
  float v[NP][VEC], r[NP][VEC];
  const int64_t first = (static_cast<int64_t>(blockIdx.x) * NP * kThreads + threadIdx.x) * VEC;
#pragma unroll
  for (int p = 0; p < NP; ++p) {
    const int64_t i = first + static_cast<int64_t>(p) * kThreads * VEC;
    if (i >= count) break;
    load_row<T, true>(x, i, count, v[p]);
    if constexpr (RES) load_row<T, true>(res, i, count, r[p]);
  }
#pragma unroll
  for (int p = 0; p < NP; ++p) {
    const int64_t i = first + static_cast<int64_t>(p) * kThreads * VEC;
    if (i >= count) break;
#pragma unroll
    for (int q = 0; q < VEC; q += 4) {
      uint32_t w[4];
      philox(static_cast<uint64_t>(i + q) >> 2, offset, seed, w);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float d = w[j] >= threshold ? v[p][q + j] * scale : 0.0f;
        v[p][q + j] = RES ? r[p][q + j] + d : d;
      }
    }
    store_row<T, true>(y, i, count, v[p]);
  }
}

template <typename T, bool RES>
void run(const void* x, const void* res, uint64_t threshold, float scale, uint64_t seed,
         uint64_t offset, const uint64_t* step, void* y, int64_t count, hipStream_t st) {
  constexpr int NP = 2;
  const int64_t per = static_cast<int64_t>(kThreads) * Row<T>::VEC * NP;
  k_dropout<T, RES, NP><<<static_cast<uint32_t>((count + per - 1) / per), kThreads, 0, st>>>(
      static_cast<const T*>(x), static_cast<const T*>(res), threshold, scale, seed, offset, step,
      static_cast<T*>(y), count);
}

}  // namespace
}  // namespace spc

using namespace spc;

extern "C" int spconv_dropout_forward(int dt, const void* x, const void* residual, double p,
                                      uint64_t seed, uint64_t offset, const uint64_t* step, void* y,
                                      int64_t count, void* stream) {
  // (2^34 elements: what one launch holds)
  if (!dtype_ok(dt) || !(p >= 0.0 && p < 1.0) || count < 0 || count >= (1ll << 34) ||
      !ptr_ok(x, count, elem_bytes(dt)) || !ptr_ok(y, count, elem_bytes(dt)) ||
      !aligned_to(residual, elem_bytes(dt)) || !aligned_to(step, 8))
    return SPCONV_EINVAL;
  if (count == 0) return SPCONV_OK;
  // up to 2^32 itself, which drops everything
  const uint64_t threshold = static_cast<uint64_t>(std::nearbyint(p * 4294967296.0));
  const float scale = static_cast<float>(1.0 / (1.0 - p));
  const auto go = [&](auto* type, auto res) {
    run<std::remove_pointer_t<decltype(type)>, res.value>(x, residual, threshold, scale, seed,
                                                          offset, step, y, count,
                                                          static_cast<hipStream_t>(stream));
  };
  bf16_t* const b = nullptr;
  float* const f = nullptr;
  if (dt == SPCONV_BF16) residual ? go(b, std::true_type{}) : go(b, std::false_type{});
  else residual ? go(f, std::true_type{}) : go(f, std::false_type{});
  return launched();
}

extern "C" int spconv_dropout_backward(int dt, const void* dy, double p, uint64_t seed,
                                       uint64_t offset, const uint64_t* step, void* dx,
                                       int64_t count, void* stream) {
  return spconv_dropout_forward(dt, dy, nullptr, p, seed, offset, step, dx, count, stream);
}
