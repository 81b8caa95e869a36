// Device-side helpers shared by the attention kernels.
#pragma once

#include "common.hpp"
#include "kernels.hpp"

namespace starq {

namespace {

typedef short v4i16_t __attribute__((ext_vector_type(4)));
#define STARQ_LDS __attribute__((address_space(3)))

constexpr int kQRows = 32;        // query rows per MFMA tile
constexpr int kBlockRows = kAttnBlockRows;  // query rows per workgroup

__device__ __attribute__((aligned(256))) uint32_t g_attn_zero[64];

__device__ __forceinline__ void wait_vm_all() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((7 << 4) | (15 << 8));  // vmcnt(0)
  asm volatile("" ::: "memory");
}
__device__ __forceinline__ uint32_t lds_addr(const void* p) {
  return __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(reinterpret_cast<uintptr_t>(p)));
}

// a in F(i, j): star (law 0) {i, j}; dense (law 1) every group; tensor power
// (law 2) every bit of a equal to that bit of i or of j.
__device__ __forceinline__ bool attn_in_group(int law, int i, int j, int a) {
  if (law == 1) return true;
  if (law == 2) return ((a ^ i) & (a ^ j)) == 0;
  return a == i || a == j;
}
__device__ __forceinline__ uint32_t attn_fmask(int law, int q, int i, int j) {
  uint32_t f = 0;
  for (int a = 0; a < q; ++a)
    if (attn_in_group(law, i, j, a)) f |= 1u << a;
  return f;
}

typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));

// max / sum of a value and its partner lane l ^ 32 (v_permlane32_swap; both
// lanes get the same result)
__device__ __forceinline__ float max_xor32(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_xor32(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Two fp32 values rounded to bf16 (nearest even) and packed, low half first:
// one v_cvt_pk_bf16_f32.
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_t){a, b}, bf16x2_t));
}

// ---- work items of a pack (see PackView) --------------------------------------

__device__ __forceinline__ bool pack_matches(const PackView& v, int32_t T, int32_t n_seq, int32_t q) {
  const int4 h = *reinterpret_cast<const int4*>(v.head);  // (one load)
  return (h.x == kPackMagic) & (h.y == T) & (h.z == n_seq) & (h.w == q);
}

// This workgroup's head and record (see PackGrid); false: none.
__device__ __forceinline__ bool pack_item(const PackView& v, int32_t heads, int& h, int32_t& k) {
  const PackGrid g = pack_grid(heads);
  const int32_t i = blockIdx.x >> 3, unit = (blockIdx.x & 7) * g.per_xcd + i % g.per_xcd;
  h = unit / g.cuts;
  k = i / g.per_xcd * g.cuts + unit % g.cuts;
  return k < v.head[4];
}

// Zeros for the rows of a chunk of kPackClearRows rows that no work item
// writes: those whose type is out of range and, if `rest`, those outside every
// sequence.  `width` elements a row (a multiple of 8); lse rows get -inf.
__device__ __forceinline__ void pack_clear_rows(const PackView& v, int32_t T, int32_t chunk, int32_t rest, void* out,
                                                int dtype, int32_t width, float* lse = nullptr, int32_t heads = 0) {
  const int lane = threadIdx.x & 63;
  const int32_t wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  const int32_t lo = chunk * kPackClearRows, hi = min(T, lo + kPackClearRows);
  for (int32_t r0 = lo + 64 * wave; r0 < hi; r0 += 64 * waves) {
    const int m = r0 + lane < hi ? v.mark[r0 + lane] : 1;
    uint64_t todo = __ballot(m == 0 || (m == 2 && rest));
    while (todo) {
      const int64_t r = r0 + __ffsll(static_cast<unsigned long long>(todo)) - 1;
      todo &= todo - 1;
      if (out) {
        const int64_t n16 = static_cast<int64_t>(width) * (dtype == 0 ? 4 : 2) / 16;
        uint4* row = static_cast<uint4*>(out) + r * n16;
        for (int64_t x = lane; x < n16; x += 64) row[x] = make_uint4(0, 0, 0, 0);
      }
      if (lse)
        for (int x = lane; x < heads; x += 64) lse[static_cast<int64_t>(x) * T + r] = -INFINITY;
    }
  }
}

}  // namespace

}  // namespace starq
