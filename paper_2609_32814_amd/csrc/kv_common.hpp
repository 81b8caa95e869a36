// Device-side reading of the paged key-value cache's 8-bit rows (see KvPages).
#pragma once

#include "common.hpp"
#include "kernels.hpp"

namespace starq {

namespace {

// 2^(b - 127), NaN for 255
__device__ __forceinline__ float kv_scale(uint32_t b) { return __uint_as_float(b == 255 ? 0x7fc00000u : b << 23); }

// Four 8-bit elements as floats (exact).
template <int TYPE>
__device__ __forceinline__ void kv_unpack4(uint32_t w, float* y) {
  if constexpr (TYPE == kKvE4m3) {
    const auto a = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w), false);
    const auto b = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w), true);
    y[0] = a[0];
    y[1] = a[1];
    y[2] = b[0];
    y[3] = b[1];
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = static_cast<float>(static_cast<int>(w << (24 - 8 * e)) >> 24);
  }
}

}  // namespace

}  // namespace starq
