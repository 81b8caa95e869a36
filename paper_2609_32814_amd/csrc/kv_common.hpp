// Device-side reading of the paged key-value cache's 8-bit rows (see KvPages).
#pragma once

#include "attn_common.hpp"

namespace starq {

namespace {

// 2^(b - 127) of scale byte e of a word, zero for byte 0.  Byte 255 is infinity,
// and a row that has it holds zeros: every product with it is NaN, as the row's
// values are.
__device__ __forceinline__ float kv_scale(uint32_t w, int e) {
  return __uint_as_float((e < 3 ? w << (23 - 8 * e) : w >> 1) & 0x7f800000u);
}

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

// Four 8-bit elements as bf16 (exact), two words.
template <int TYPE>
__device__ __forceinline__ uint2 kv_bf16x4(uint32_t w) {
  if constexpr (TYPE == kKvE4m3) {
    return make_uint2(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(static_cast<int>(w), 1.0f, false)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(static_cast<int>(w), 1.0f, true)));
  } else {
    float y[4];
    kv_unpack4<TYPE>(w, y);
    return make_uint2(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]));
  }
}

}  // namespace

}  // namespace starq
