// Elements on their way into a cache.
#pragma once
#include "lfps_internal.h"

#include <type_traits>

namespace lfps {

// Eight elements as they are stored: TS of the new rows, TC of the cache.
template <typename TS, typename TC>
struct Convert8 {
  static_assert(sizeof(TS) == sizeof(TC), "");
  __device__ __forceinline__ static void move(const TS* from, TC* to) {
#pragma unroll
    for (int u = 0; u < (int)sizeof(TS) / 2; ++u) reinterpret_cast<u32x4*>(to)[u] = reinterpret_cast<const u32x4*>(from)[u];
  }
};
template <>
struct Convert8<uint16_t, uint8_t> {
  __device__ __forceinline__ static void move(const uint16_t* from, uint8_t* to) {
    const u32x4 w = *reinterpret_cast<const u32x4*>(from);
    u32x2 r;
    auto kept = [](float x) { return x != x ? x : fminf(fmaxf(x, -448.f), 448.f); };
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      int v = __builtin_amdgcn_cvt_pk_fp8_f32(kept(bf16_lo(w[2 * u])), kept(bf16_hi(w[2 * u])), 0, false);
      v = __builtin_amdgcn_cvt_pk_fp8_f32(kept(bf16_lo(w[2 * u + 1])), kept(bf16_hi(w[2 * u + 1])), v, true);
      r[u] = (uint32_t)v;
    }
    *reinterpret_cast<u32x2*>(to) = r;
  }
};

// Eight fp32 values, rounded once to the type they are stored in (nearest even; FP8: beyond +-448 and infinities +-448, NaN stays NaN).
template <typename T>
__device__ __forceinline__ void store8(T* to, const float (&x)[8]) {
  if constexpr (std::is_same<T, float>::value) {
    reinterpret_cast<f32x4*>(to)[0] = f32x4{x[0], x[1], x[2], x[3]};
    reinterpret_cast<f32x4*>(to)[1] = f32x4{x[4], x[5], x[6], x[7]};
  } else if constexpr (std::is_same<T, uint8_t>::value) {
    auto kept = [](float y) { return y != y ? y : fminf(fmaxf(y, -448.f), 448.f); };
    u32x2 r;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      int v = __builtin_amdgcn_cvt_pk_fp8_f32(kept(x[4 * u]), kept(x[4 * u + 1]), 0, false);
      v = __builtin_amdgcn_cvt_pk_fp8_f32(kept(x[4 * u + 2]), kept(x[4 * u + 3]), v, true);
      r[u] = (uint32_t)v;
    }
    *reinterpret_cast<u32x2*>(to) = r;
  } else {
    typedef typename std::conditional<std::is_same<T, uint16_t>::value, __bf16, _Float16>::type Elem;
    typedef Elem Elem8 __attribute__((ext_vector_type(8)));
    Elem8 y;
#pragma unroll
    for (int c = 0; c < 8; ++c) y[c] = (Elem)x[c];
    *reinterpret_cast<Elem8*>(to) = y;
  }
}

}  // namespace lfps
