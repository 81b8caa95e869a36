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
// A workgroup takes TG tokens: it looks each one's place up once, then goes
// through the rows of all their heads, 16 bytes of a page row to a lane, the
// rows of one head's tokens side by side (they are neighbours in the page).  A
// row's largest magnitude is joined by lane exchanges.  Both kernels are bound
// by memory: every row is read once and written once.  40000 tokens, 8 heads of
// 128, from e4m3: 58 us, 4.3 TB/s; 16411 tokens to e4m3 and back 19 us each
// (in cache); 64 tokens: 3.6 us, a launch and the look-up of a page.
#include "attn_common.hpp"
#include "kv_common.hpp"

namespace starq {

namespace {

constexpr int kThreads = 256;

// Bounds of the sequences count as the pack's plan counts them: no lower than an
// earlier one or 0, no higher than T.  So the first bound above a token ends
// its sequence, whatever order they are in, and a search by halving would not
// do.  Wavefront w looks through bounds 256 w .. 256 w + 255 of every 1024, four
// a lane asked for at once, until one lies above all TG tokens; lane j ends
// with the index of its first one above token t0 + j (INT32_MAX: none).  A
// token each to int8, 12 heads of 64, us so and by halving: 64 sequences 3.6 and
// 3.8, 4096 8.5 and 8.8, 16384 25.5 and 20.4.
template <int TG>
__device__ __forceinline__ int32_t first_above(const int32_t* cu, int32_t n_seq, int32_t t0, int lane, int wave) {
  int32_t first = INT32_MAX;
  for (int64_t k0 = 256 * wave; k0 <= n_seq; k0 += 4 * kThreads) {
    int32_t c[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) c[u] = k0 + 64 * u + lane <= n_seq ? cu[k0 + 64 * u + lane] : INT32_MIN;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int32_t k = static_cast<int32_t>(k0) + 64 * u;
      const uint64_t any = __ballot(c[u] > t0);
      if (any == 0) continue;
      const int at = __builtin_ctzll(any);
      if (__builtin_amdgcn_readlane(c[u], at) > t0 + TG - 1) {  // one sequence holds them all
        first = min(first, k + at);
        continue;
      }
#pragma unroll
      for (int j = 0; j < TG; ++j) {
        const uint64_t m = __ballot(c[u] > t0 + j);
        if (lane == j) first = min(first, m ? k + __builtin_ctzll(m) : INT32_MAX);
      }
    }
    if (__ballot(lane < TG && first == INT32_MAX) == 0) break;
  }
  return first;
}

// Where the entry of token t < T lies, `end` the first bound above it: the row
// index (page n_kv + head) page_size + place of its head 0, or -1 (no such
// entry), -2 (outside every sequence).
__device__ __forceinline__ int64_t find_row(const KvPages& kv, const int32_t* cu, const int32_t* cache_len, int32_t T, int32_t t,
                                            int32_t end) {
  if (end == 0 || end > kv.B) return -2;
  const int64_t pos = static_cast<int64_t>(cache_len[end - 1]) - (min(cu[end], T) - t);
  if (pos < 0 || (pos >> kv.page_shift) >= kv.max_pages) return -1;
  const int32_t page = kv.table[static_cast<int64_t>(end - 1) * kv.max_pages + (pos >> kv.page_shift)];
  if (static_cast<unsigned>(page) >= static_cast<unsigned>(kv.n_pages)) return -1;
  return ((static_cast<int64_t>(page) * kv.n_kv) << kv.page_shift) + (pos & ((1 << kv.page_shift) - 1));
}

// Elements of a row that a lane holds: 16 bytes of the page.
template <int TYPE>
constexpr int lane_elems() { return TYPE == kKvBf16 ? 8 : 16; }

// 16 elements of a row (in[0], in[1]) to 16 bytes; LANES lanes hold the row.
// Returns the scale byte.
template <int TYPE, int LANES>
__device__ __forceinline__ int quantise(const uint4* in, uint4& out) {
  const uint32_t w[8] = {in[0].x, in[0].y, in[0].z, in[0].w, in[1].x, in[1].y, in[1].z, in[1].w};
  uint32_t top = 0;  // largest magnitude as bits: their order is that of the values, NaN above all
#pragma unroll
  for (int e = 0; e < 8; ++e) top = max(top, max((w[e] << 16) & 0x7fff0000u, w[e] & 0x7fff0000u));
#pragma unroll
  for (int d = LANES / 2; d > 0; d >>= 1) top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), d, LANES)));
  out = make_uint4(0, 0, 0, 0);
  if (top >= 0x7f800000u) return 255;
  // top = 1.f 2^k against 1.75 2^8 or 1.984375 2^6
  constexpr uint32_t kFrac = TYPE == kKvE4m3 ? 0x600000u : 0x7e0000u;
  constexpr int kExp = TYPE == kKvE4m3 ? 8 : 6;
  const int scale = max(1, static_cast<int>(top >> 23) - kExp + ((top & 0x7fffffu) > kFrac ? 1 : 0));
  const float inv = __uint_as_float(static_cast<uint32_t>(254 - scale) << 23);
  uint32_t v[4];
#pragma unroll
  for (int x = 0; x < 4; ++x) {
    const float y0 = __uint_as_float(w[2 * x] << 16) * inv, y1 = __uint_as_float(w[2 * x] & 0xffff0000u) * inv;
    const float y2 = __uint_as_float(w[2 * x + 1] << 16) * inv, y3 = __uint_as_float(w[2 * x + 1] & 0xffff0000u) * inv;
    if constexpr (TYPE == kKvE4m3) {
      v[x] = static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(y2, y3, __builtin_amdgcn_cvt_pk_fp8_f32(y0, y1, 0, false), true));
    } else {
      auto byte = [](float y) { return static_cast<uint32_t>(static_cast<int>(__builtin_rintf(y))) & 0xffu; };
      v[x] = byte(y0) | byte(y1) << 8 | byte(y2) << 16 | byte(y3) << 24;
    }
  }
  out = make_uint4(v[0], v[1], v[2], v[3]);
  return scale;
}

// The places of the workgroup's TG tokens, then `each(row, token, head, c)` for
// every row of them: its place (see find_row), and which of its lanes this is.
template <int DH, int TYPE, int TG, class Each>
__device__ __forceinline__ void for_rows(const KvPages& kv, const int32_t* cu, const int32_t* cache_len, int32_t T, Each each) {
  constexpr int LANES = DH / lane_elems<TYPE>(), RP = kThreads / LANES;
  constexpr int kWaves = kThreads / 64;
  __shared__ int64_t place[TG];
  __shared__ int32_t above[kWaves][TG];
  const int64_t t0 = static_cast<int64_t>(blockIdx.x) * TG;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int32_t first = first_above<TG>(cu, kv.B, static_cast<int32_t>(t0), lane, wave);
  if (lane < TG) above[wave][lane] = first;
  __syncthreads();
  if (threadIdx.x < TG) {
    int32_t end = first;
#pragma unroll
    for (int w = 1; w < kWaves; ++w) end = min(end, above[w][threadIdx.x]);
    const int64_t t = t0 + threadIdx.x;
    place[threadIdx.x] = t < T ? find_row(kv, cu, cache_len, T, static_cast<int32_t>(t), end) : -3;
  }
  __syncthreads();
  const int c = threadIdx.x % LANES;
#pragma unroll 4
  for (int32_t r = threadIdx.x / LANES; r < TG * kv.n_kv; r += RP) {
    const int32_t head = r / TG;
    int64_t row = place[r % TG];
    if (row >= 0) row += static_cast<int64_t>(head) << kv.page_shift;
    each(row, t0 + r % TG, head, c);
  }
}

// blockIdx.y 0: keys, 1: values
template <int DH, int TYPE, int TG>
__global__ __launch_bounds__(kThreads) void kv_append_kernel(const KvPages kv, const int32_t* cu, const int32_t* cache_len,
                                                             int32_t T, const uint16_t* K, const uint16_t* V) {
  constexpr int LE = lane_elems<TYPE>();
  const uint16_t* src = blockIdx.y ? V : K;
  uint4* pages = static_cast<uint4*>(blockIdx.y ? kv.V : kv.K);
  uint8_t* scales = blockIdx.y ? kv.v_scale : kv.k_scale;
  for_rows<DH, TYPE, TG>(kv, cu, cache_len, T, [&](int64_t row, int64_t t, int32_t head, int c) {
    if (row < 0) return;  // (a row's lanes together)
    const uint4* in = reinterpret_cast<const uint4*>(src + (t * kv.n_kv + head) * DH + LE * c);
    uint4* to = pages + row * (DH / LE) + c;
    if constexpr (TYPE == kKvBf16) {
      *to = *in;
    } else {
      const uint4 w[2] = {in[0], in[1]};
      uint4 out;
      const int scale = quantise<TYPE, DH / LE>(w, out);
      *to = out;
      if (c == 0) scales[row] = static_cast<uint8_t>(scale);
    }
  });
}

template <int DH, int TYPE, int TG>
__global__ __launch_bounds__(kThreads) void kv_read_kernel(const KvPages kv, const int32_t* cu, const int32_t* cache_len,
                                                           int32_t T, uint16_t* K, uint16_t* V, int32_t clear_rest) {
  constexpr int LE = lane_elems<TYPE>();
  uint16_t* dst = blockIdx.y ? V : K;
  const uint4* pages = static_cast<const uint4*>(blockIdx.y ? kv.V : kv.K);
  const uint8_t* scales = blockIdx.y ? kv.v_scale : kv.k_scale;
  for_rows<DH, TYPE, TG>(kv, cu, cache_len, T, [&](int64_t row, int64_t t, int32_t head, int c) {
    if (row == -3 || (row == -2 && !clear_rest)) return;
    uint4* to = reinterpret_cast<uint4*>(dst + (t * kv.n_kv + head) * DH + LE * c);
    uint4 in = make_uint4(0, 0, 0, 0);
    if (row >= 0) in = pages[row * (DH / LE) + c];
    if constexpr (TYPE == kKvBf16) {
      *to = in;
    } else {
      const float s = row >= 0 ? kv_scale(scales[row], 0) : 0.f;
      const uint32_t w[4] = {in.x, in.y, in.z, in.w};
      uint32_t o[8];
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        float y[4];
        kv_unpack4<TYPE>(w[x], y);
        o[2 * x] = pack_bf16(y[0] * s, y[1] * s);
        o[2 * x + 1] = pack_bf16(y[2] * s, y[3] * s);
      }
      to[0] = make_uint4(o[0], o[1], o[2], o[3]);
      to[1] = make_uint4(o[4], o[5], o[6], o[7]);
    }
  });
}

// 16 tokens a workgroup; 4 where that would leave CUs without one.  To int8, 64
// sequences, 12 heads of 64, us with 4 and with 16: 64 tokens 3.6 and 4.9, 2048
// tokens 4.6 and 5.1, 4096 6.0 and 6.3, 8192 10.1 and 9.1 (and back 3.6 and
// 4.6, 5.2 and 5.5, 7.1 and 7.1, 10.6 and 10.2).
constexpr int kMany = 16, kFew = 4;
bool few_tokens(int32_t T, int32_t cus) { return T < cus * kMany; }

template <int DH, int TYPE, int TG>
hipError_t append_tg(const KvPages& kv, const int32_t* cu, const int32_t* len, int32_t T, const void* K, const void* V,
                     hipStream_t stream) {
  hipLaunchKernelGGL((kv_append_kernel<DH, TYPE, TG>), dim3((T + TG - 1) / TG, 2), dim3(kThreads), 0, stream, kv, cu, len, T,
                     static_cast<const uint16_t*>(K), static_cast<const uint16_t*>(V));
  return hipGetLastError();
}
template <int DH, int TYPE>
hipError_t append(const KvPages& kv, const int32_t* cu, const int32_t* len, int32_t T, const void* K, const void* V,
                  int32_t cus, hipStream_t stream) {
  return few_tokens(T, cus) ? append_tg<DH, TYPE, kFew>(kv, cu, len, T, K, V, stream)
                            : append_tg<DH, TYPE, kMany>(kv, cu, len, T, K, V, stream);
}
template <int DH, int TYPE, int TG>
hipError_t read_tg(const KvPages& kv, const int32_t* cu, const int32_t* len, int32_t T, void* K, void* V, int32_t clear_rest,
                   hipStream_t stream) {
  hipLaunchKernelGGL((kv_read_kernel<DH, TYPE, TG>), dim3((T + TG - 1) / TG, 2), dim3(kThreads), 0, stream, kv, cu, len, T,
                     static_cast<uint16_t*>(K), static_cast<uint16_t*>(V), clear_rest);
  return hipGetLastError();
}
template <int DH, int TYPE>
hipError_t read(const KvPages& kv, const int32_t* cu, const int32_t* len, int32_t T, void* K, void* V, int32_t clear_rest,
                int32_t cus, hipStream_t stream) {
  return few_tokens(T, cus) ? read_tg<DH, TYPE, kFew>(kv, cu, len, T, K, V, clear_rest, stream)
                            : read_tg<DH, TYPE, kMany>(kv, cu, len, T, K, V, clear_rest, stream);
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
                            const void* V, int32_t cus, hipStream_t stream) {
  STARQ_KV_DISPATCH(append, kv, cu, cache_len, T, K, V, cus, stream)
}

hipError_t launch_kv_read(const KvPages& kv, const int32_t* cu, const int32_t* cache_len, int32_t T, void* K, void* V,
                          int32_t clear_rest, int32_t cus, hipStream_t stream) {
  STARQ_KV_DISPATCH(read, kv, cu, cache_len, T, K, V, clear_rest, cus, stream)
}

}  // namespace starq
