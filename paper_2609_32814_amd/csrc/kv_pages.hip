// The paged key-value cache: rows of new keys and values are written into its
// pages, quantised to 8 bits where the pages hold those, and read back.
//
// A row (one token, one head) in 8 bits is its elements times a power of two
// 2^-e, rounded to nearest even, with e the least at which its largest
// magnitude fits the type (448 for e4m3, 127 for int8; e >= -126), kept as the
// byte e + 127.  A power of two makes the scaling, the rounding's input and
// the value read back (at most 8 significant bits) exact, also in bf16; e4m3
// loses nothing by it, int8 at most one bit of its seven.  A row that holds a
// NaN or an infinity is kept as scale byte 255 and reads back as NaN.
//
// head_dim / 8 lanes take a row, 16 bytes of bf16 each; the row's largest
// magnitude is joined by lane exchanges.  Both kernels are bound by memory:
// every row is read once and written once.
#include "attn_common.hpp"
#include "kv_common.hpp"

namespace starq {

namespace {

constexpr int kThreads = 256;

// Where token t's entry lies: the row index (page n_kv + head) page_size +
// place of its head 0, or -1 (no such entry), -2 (outside every sequence).
__device__ __forceinline__ int64_t find_row(const KvPages& kv, const int32_t* cu, const int32_t* cache_len, int32_t t) {
  if (t < cu[0] || t >= cu[kv.B]) return -2;
  int32_t lo = 0, hi = kv.B;  // cu[lo] <= t < cu[hi]
  while (hi - lo > 1) {
    const int32_t mid = (lo + hi) >> 1;
    if (cu[mid] <= t) lo = mid;
    else hi = mid;
  }
  const int64_t pos = static_cast<int64_t>(cache_len[lo]) - (static_cast<int64_t>(cu[lo + 1]) - t);
  if (pos < 0 || (pos >> kv.page_shift) >= kv.max_pages) return -1;
  const int32_t page = kv.table[static_cast<int64_t>(lo) * kv.max_pages + (pos >> kv.page_shift)];
  if (static_cast<unsigned>(page) >= static_cast<unsigned>(kv.n_pages)) return -1;
  return ((static_cast<int64_t>(page) * kv.n_kv) << kv.page_shift) + (pos & ((1 << kv.page_shift) - 1));
}

// 8 elements of a row to 8 bytes; LANES lanes hold the row.  Returns the scale byte.
template <int TYPE, int LANES>
__device__ __forceinline__ int quantise(const uint4& in, uint2& out) {
  const uint32_t w[4] = {in.x, in.y, in.z, in.w};
  uint32_t top = 0;  // largest magnitude as bits: their order is that of the values, NaN above all
#pragma unroll
  for (int e = 0; e < 4; ++e) top = max(top, max((w[e] << 16) & 0x7fff0000u, w[e] & 0x7fff0000u));
#pragma unroll
  for (int d = LANES / 2; d > 0; d >>= 1) top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), d, LANES)));
  out = make_uint2(0, 0);
  if (top >= 0x7f800000u) return 255;
  // top = 1.f 2^k against 1.75 2^8 or 1.984375 2^6
  constexpr uint32_t kFrac = TYPE == kKvE4m3 ? 0x600000u : 0x7e0000u;
  constexpr int kExp = TYPE == kKvE4m3 ? 8 : 6;
  const int scale = max(1, static_cast<int>(top >> 23) - kExp + ((top & 0x7fffffu) > kFrac ? 1 : 0));
  const float inv = __uint_as_float(static_cast<uint32_t>(254 - scale) << 23);
  float y[8];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    y[2 * e] = __uint_as_float(w[e] << 16) * inv;
    y[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u) * inv;
  }
  if constexpr (TYPE == kKvE4m3) {
    int a = 0, b = 0;
    a = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], a, false);
    a = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], a, true);
    b = __builtin_amdgcn_cvt_pk_fp8_f32(y[4], y[5], b, false);
    b = __builtin_amdgcn_cvt_pk_fp8_f32(y[6], y[7], b, true);
    out = make_uint2(a, b);
  } else {
    uint32_t v[2] = {0, 0};
#pragma unroll
    for (int e = 0; e < 8; ++e)
      v[e / 4] |= (static_cast<uint32_t>(static_cast<int>(__builtin_rintf(y[e]))) & 0xffu) << (8 * (e % 4));
    out = make_uint2(v[0], v[1]);
  }
  return scale;
}

// blockIdx.y 0: keys, 1: values
template <int DH, int TYPE>
__global__ __launch_bounds__(kThreads) void kv_append_kernel(const KvPages kv, const int32_t* cu, const int32_t* cache_len,
                                                             int32_t T, const uint16_t* K, const uint16_t* V) {
  constexpr int LANES = DH / 8;
  const int64_t r = (static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x) / LANES;  // token n_kv + head
  const int c = threadIdx.x % LANES;
  if (r >= static_cast<int64_t>(T) * kv.n_kv) return;  // (a row's lanes together)
  const int32_t t = static_cast<int32_t>(r / kv.n_kv), head = static_cast<int32_t>(r % kv.n_kv);
  const uint4 in = *reinterpret_cast<const uint4*>((blockIdx.y ? V : K) + r * DH + 8 * c);
  int64_t row = find_row(kv, cu, cache_len, t);
  if (row < 0) return;
  row += static_cast<int64_t>(head) << kv.page_shift;
  void* pages = blockIdx.y ? kv.V : kv.K;
  if constexpr (TYPE == kKvBf16) {
    *reinterpret_cast<uint4*>(static_cast<uint16_t*>(pages) + row * DH + 8 * c) = in;
  } else {
    uint2 out;
    const int scale = quantise<TYPE, LANES>(in, out);
    *reinterpret_cast<uint2*>(static_cast<uint8_t*>(pages) + row * DH + 8 * c) = out;
    if (c == 0) (blockIdx.y ? kv.v_scale : kv.k_scale)[row] = static_cast<uint8_t>(scale);
  }
}

template <int DH, int TYPE>
__global__ __launch_bounds__(kThreads) void kv_read_kernel(const KvPages kv, const int32_t* cu, const int32_t* cache_len,
                                                           int32_t T, uint16_t* K, uint16_t* V, int32_t clear_rest) {
  constexpr int LANES = DH / 8;
  const int64_t r = (static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x) / LANES;
  const int c = threadIdx.x % LANES;
  if (r >= static_cast<int64_t>(T) * kv.n_kv) return;
  const int32_t t = static_cast<int32_t>(r / kv.n_kv), head = static_cast<int32_t>(r % kv.n_kv);
  int64_t row = find_row(kv, cu, cache_len, t);
  if (row == -2 && !clear_rest) return;
  uint4 out = make_uint4(0, 0, 0, 0);
  if (row >= 0) {
    row += static_cast<int64_t>(head) << kv.page_shift;
    const void* pages = blockIdx.y ? kv.V : kv.K;
    if constexpr (TYPE == kKvBf16) {
      out = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(pages) + row * DH + 8 * c);
    } else {
      const uint2 in = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(pages) + row * DH + 8 * c);
      const float s = kv_scale((blockIdx.y ? kv.v_scale : kv.k_scale)[row]);
      float y[8];
      kv_unpack4<TYPE>(in.x, y);
      kv_unpack4<TYPE>(in.y, y + 4);
      out = make_uint4(pack_bf16(y[0] * s, y[1] * s), pack_bf16(y[2] * s, y[3] * s), pack_bf16(y[4] * s, y[5] * s),
                       pack_bf16(y[6] * s, y[7] * s));
    }
  }
  *reinterpret_cast<uint4*>((blockIdx.y ? V : K) + r * DH + 8 * c) = out;
}

unsigned rows_grid(const KvPages& kv, int32_t T) {
  const int64_t lanes = static_cast<int64_t>(T) * kv.n_kv * (kv.head_dim / 8);
  return static_cast<unsigned>((lanes + kThreads - 1) / kThreads);
}

template <int DH, int TYPE>
hipError_t append(const KvPages& kv, const int32_t* cu, const int32_t* len, int32_t T, const void* K, const void* V,
                  hipStream_t stream) {
  hipLaunchKernelGGL((kv_append_kernel<DH, TYPE>), dim3(rows_grid(kv, T), 2), dim3(kThreads), 0, stream, kv, cu, len, T,
                     static_cast<const uint16_t*>(K), static_cast<const uint16_t*>(V));
  return hipGetLastError();
}
template <int DH, int TYPE>
hipError_t read(const KvPages& kv, const int32_t* cu, const int32_t* len, int32_t T, void* K, void* V, int32_t clear_rest,
                hipStream_t stream) {
  hipLaunchKernelGGL((kv_read_kernel<DH, TYPE>), dim3(rows_grid(kv, T), 2), dim3(kThreads), 0, stream, kv, cu, len, T,
                     static_cast<uint16_t*>(K), static_cast<uint16_t*>(V), clear_rest);
  return hipGetLastError();
}

}  // namespace

#define STARQ_KV_DISPATCH(fn, ...)                                                                                     \
  switch (kv.type) {                                                                                                   \
    case kKvBf16: return kv.head_dim == 64 ? fn<64, kKvBf16>(__VA_ARGS__) : fn<128, kKvBf16>(__VA_ARGS__);             \
    case kKvE4m3: return kv.head_dim == 64 ? fn<64, kKvE4m3>(__VA_ARGS__) : fn<128, kKvE4m3>(__VA_ARGS__);             \
    case kKvInt8: return kv.head_dim == 64 ? fn<64, kKvInt8>(__VA_ARGS__) : fn<128, kKvInt8>(__VA_ARGS__);             \
    default: return hipErrorInvalidValue;                                                                              \
  }

hipError_t launch_kv_append(const KvPages& kv, const int32_t* cu, const int32_t* cache_len, int32_t T, const void* K,
                            const void* V, hipStream_t stream) {
  STARQ_KV_DISPATCH(append, kv, cu, cache_len, T, K, V, stream)
}

hipError_t launch_kv_read(const KvPages& kv, const int32_t* cu, const int32_t* cache_len, int32_t T, void* K, void* V,
                          int32_t clear_rest, hipStream_t stream) {
  STARQ_KV_DISPATCH(read, kv, cu, cache_len, T, K, V, clear_rest, stream)
}

}  // namespace starq
