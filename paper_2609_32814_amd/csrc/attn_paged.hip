// Attention of one new token per sequence over a paged key-value cache.
//
// The work is the list of (sequence, key/value head, slice of up to 16 of its
// query heads), each with its tiles of 128 keys.  `wgs` workgroups take equal
// contiguous shares of that list, whatever the sequences' lengths: a long
// sequence is split over many workgroups, and a workgroup may end one sequence
// and begin the next.  Each piece of a pair keeps a running maximum and sum; a
// piece that is the whole pair is written out, the others are joined by the
// second launch in the order of their workgroups.
//
// A wavefront takes 32 keys of a tile, with 16 x 16 x 32 bf16 products whose
// columns are the query heads (padded to 16: the products are far from their
// limit, the cache's bytes bound the kernel):
//   S = K Q^T: lane l brings 8 features of key row l % 16 straight from memory.
//       Row r of half t stands for key 8 (r / 4) + 4 t + r % 4, so that a lane
//       ends with the scores of 8 consecutive keys 8 (l / 16) + 0..7 of head
//       l % 16 ...
//   O^T += V^T P: ... which is the operand P of the second product as it lies.
//       For V^T lane l loads DH / 16 features from (DH / 16) (l % 16) on of
//       those 8 keys (whole rows over 16 lanes) and turns the block in its
//       registers; row r of product e stands for feature (DH / 16) r + e.
// 8-bit rows become bf16 exactly; a key's scale goes into its score, a value's
// into its probability.  A cell of 8 features that a key's type does not
// select, a key behind the sequence's end, of a type out of range or in a page
// out of range is not read, and zeros stand in its place.
#include "attn_common.hpp"
#include "kv_common.hpp"

namespace starq {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kTile = 32 * kWaves;  // keys

typedef float f32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ f32x4 mfma16(uint4 a, uint4 b, const f32x4& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}

// max / sum over the four lanes l % 16 + 16 k
__device__ __forceinline__ float max_quarters(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return max_xor32(x);
}
__device__ __forceinline__ float sum_quarters(float x) {
  x += __shfl_xor(x, 16);
  return sum_xor32(x);
}

__device__ __forceinline__ int32_t cached(const AttnPagedParams& p, int32_t b) { return max(0, min(p.cache_len[b], p.cap)); }
__device__ __forceinline__ int64_t tiles_of(int32_t len) { return (len + kTile - 1) / kTile; }

// Sums of tiles over the sequences: all of them and those before `b`, or with
// b < 0 only all.
template <int THREADS>
__device__ __forceinline__ void count_tiles(const AttnPagedParams& p, int32_t b, int64_t* red, int64_t& all, int64_t& before) {
  int64_t a = 0, f = 0;
  for (int32_t x = threadIdx.x; x < p.kv.B; x += THREADS) {
    const int64_t n = tiles_of(cached(p, x));
    a += n;
    if (x < b) f += n;
  }
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) {
    a += __shfl_xor(a, d);
    f += __shfl_xor(f, d);
  }
  if ((threadIdx.x & 63) == 0) {
    red[2 * (threadIdx.x >> 6)] = a;
    red[2 * (threadIdx.x >> 6) + 1] = f;
  }
  __syncthreads();
  all = before = 0;
  for (int w = 0; w < THREADS / 64; ++w) {
    all += red[2 * w];
    before += red[2 * w + 1];
  }
}

// The rows of 32 keys as they lie in memory, for one lane.
template <int DH, int TYPE>
struct Rows {
  static constexpr int KS = DH / 32;
  static constexpr int EL = TYPE == kKvBf16 ? 2 : 1;  // bytes per element
  static constexpr int KW = 2 * EL;                   // words of 8 features
  static constexpr int VW = DH / 64 * EL;             // words of DH / 16 features
  uint32_t k[2][KS][KW];
  uint32_t v[8][VW];
  uint2 ks, vs;      // scale bytes of keys 8 (l / 16) + 0..7
  int32_t type[8];   // their types, or -1
};

template <int N>
__device__ __forceinline__ void load_words(uint32_t* to, const void* from) {
  if constexpr (N == 4) {
    const uint4 x = *static_cast<const uint4*>(from);
    to[0] = x.x, to[1] = x.y, to[2] = x.z, to[3] = x.w;
  } else if constexpr (N == 2) {
    const uint2 x = *static_cast<const uint2*>(from);
    to[0] = x.x, to[1] = x.y;
  } else {
    to[0] = *static_cast<const uint32_t*>(from);
  }
}

template <int DH, int TYPE>
__global__ __launch_bounds__(kThreads) void attn_paged_part_kernel(const AttnPagedParams p) {
  typedef Rows<DH, TYPE> R;
  constexpr int KS = R::KS, EL = R::EL, F = DH / 16;
  extern __shared__ __attribute__((aligned(16))) float wsm[];  // [wave][16][DH + 4]: O, maximum, sum
  __shared__ int64_t red[2 * kWaves];
  __shared__ int64_t at_s[2];
  __shared__ int32_t b_s;
  __shared__ uint32_t cells_s[kAttnMaxQ];
  __shared__ float scale_s[kAttnMaxQ];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l16 = lane & 15, quad = lane >> 4;
  const int q = p.q, m = DH / q, cpg = m / 8;
  const int rep = p.n_heads / p.kv.n_kv;
  const int32_t pairs = p.kv.n_kv * p.groups;  // of one sequence

  // ---- this workgroup's share
  int64_t all, unused;
  count_tiles<kThreads>(p, -1, red, all, unused);
  all *= pairs;
  const int64_t wgs = all < p.wgs ? all : p.wgs;
  if (blockIdx.x >= wgs) return;
  int64_t u = blockIdx.x * all / wgs;
  const int64_t u_end = (blockIdx.x + 1) * all / wgs;
  // the sequence that holds tile u: a running sum over chunks of sequences
  int64_t carry = 0;
  for (int32_t b0 = 0;; b0 += kThreads) {
    const int32_t b = b0 + threadIdx.x;
    const int64_t n = b < p.kv.B ? tiles_of(cached(p, b)) * pairs : 0;
    int64_t incl = n;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int64_t o = __shfl_up(incl, d);
      if (lane >= d) incl += o;
    }
    __syncthreads();
    if (lane == 63) red[wave] = incl;
    if (threadIdx.x == 0) b_s = -1;
    __syncthreads();
    int64_t chunk = 0;
    for (int w = 0; w < kWaves; ++w) {
      if (w < wave) incl += red[w];
      chunk += red[w];
    }
    if (u >= carry + incl - n && u < carry + incl) {
      b_s = b;
      at_s[0] = u - (carry + incl - n);
    }
    __syncthreads();
    if (b_s >= 0) break;
    carry += chunk;
  }
  int32_t b = b_s;
  int64_t in_seq = at_s[0];
  int32_t len = cached(p, b);
  int32_t pair = static_cast<int32_t>(in_seq / tiles_of(len));
  int32_t tile = static_cast<int32_t>(in_seq % tiles_of(len));

  // ---- pieces
  while (true) {
    const int32_t n_tiles = static_cast<int32_t>(tiles_of(len));
    const int32_t tile_end = static_cast<int32_t>(min<int64_t>(n_tiles, tile + (u_end - u)));
    const int hk = pair / p.groups, h0 = hk * rep + pair % p.groups * kPagedHeads;
    const int nh = min(kPagedHeads, rep - pair % p.groups * kPagedHeads);
    const int own = p.pos_type[len - 1];
    const bool live = static_cast<unsigned>(own) < static_cast<unsigned>(q);
    if (threadIdx.x < q) {
      const uint32_t fm = live ? attn_fmask(p.law, q, own, threadIdx.x) : 0;
      uint32_t cells = 0;
      for (int a = 0; a < q; ++a)
        if ((fm >> a) & 1u) cells |= ((1u << cpg) - 1u) << (a * cpg);
      cells_s[threadIdx.x] = cells;
      scale_s[threadIdx.x] = live ? kLog2e * __builtin_amdgcn_rsqf(static_cast<float>(__popc(fm) * m)) : 0.f;
    }
    __syncthreads();

    uint4 qf[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      qf[ks] = make_uint4(0, 0, 0, 0);
      if (l16 < nh)
        qf[ks] = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p.Q) +
                                                 (static_cast<int64_t>(b) * p.n_heads + h0 + l16) * DH + 32 * ks + 8 * quad);
    }
    f32x4 acc[F];
#pragma unroll
    for (int e = 0; e < F; ++e) acc[e] = f32x4{};
    float run_max = -INFINITY, run_sum = 0.f;

    const int32_t* table = p.kv.table + static_cast<int64_t>(b) * p.kv.max_pages;
    const int32_t page_mask = (1 << p.kv.page_shift) - 1;
    // the first row of the 8 keys from `key` on (they lie in one page), or -1
    auto row_of = [&](int32_t key) -> int64_t {
      if (key >= len) return -1;
      const int32_t page = table[key >> p.kv.page_shift];
      if (static_cast<unsigned>(page) >= static_cast<unsigned>(p.kv.n_pages)) return -1;
      return ((static_cast<int64_t>(page) * p.kv.n_kv + hk) << p.kv.page_shift) + (key & page_mask);
    };
    auto load = [&](int32_t tl, R& r) {
      const int32_t key0 = tl * kTile + 32 * wave;
      // keys: rows l16 of the halves are keys ka and ka + 4
      const int32_t blk = key0 + 8 * (l16 >> 2), ka = blk + (l16 & 3);
      const int64_t krow = row_of(blk) + (l16 & 3);
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int32_t key = ka + 4 * t;
        const int j = live && key < len ? p.pos_type[key] : -1;
        const bool ok = krow >= (l16 & 3) && static_cast<unsigned>(j) < static_cast<unsigned>(q);
        const uint32_t cells = ok ? cells_s[j] : 0u;
        const char* src = static_cast<const char*>(p.kv.K) + ((krow + 4 * t) * DH + 8 * quad) * EL;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
#pragma unroll
          for (int w = 0; w < R::KW; ++w) r.k[t][ks][w] = 0;
          if ((cells >> (4 * ks + quad)) & 1u) load_words<R::KW>(r.k[t][ks], src + 32 * ks * EL);
        }
      }
      // values, scales and types of keys vk .. vk + 7
      const int32_t vk = key0 + 8 * quad;
      const int64_t vrow = row_of(vk);
#pragma unroll
      for (int e = 0; e < 8; ++e) r.type[e] = live && vrow >= 0 && vk + e < len ? p.pos_type[vk + e] : -1;
      r.ks = r.vs = make_uint2(0, 0);
      if (TYPE != kKvBf16 && vrow >= 0) {
        r.ks = *reinterpret_cast<const uint2*>(p.kv.k_scale + vrow);
        r.vs = *reinterpret_cast<const uint2*>(p.kv.v_scale + vrow);
      }
      const char* src = static_cast<const char*>(p.kv.V) + (vrow * DH + F * l16) * EL;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
#pragma unroll
        for (int w = 0; w < R::VW; ++w) r.v[e][w] = 0;
        if (static_cast<unsigned>(r.type[e]) < static_cast<unsigned>(q)) load_words<R::VW>(r.v[e], src + e * DH * EL);
      }
    };
    auto compute = [&](const R& r) {
      f32x4 s[2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        s[t] = f32x4{};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          uint4 a;
          if constexpr (TYPE == kKvBf16) {
            a = make_uint4(r.k[t][ks][0], r.k[t][ks][1], r.k[t][ks][2], r.k[t][ks][3]);
          } else {
            float y[8];
            kv_unpack4<TYPE>(r.k[t][ks][0], y);
            kv_unpack4<TYPE>(r.k[t][ks][1], y + 4);
            a = make_uint4(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]), pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7]));
          }
          s[t] = mfma16(a, qf[ks], s[t]);
        }
      }
      float sc[8], bm = -INFINITY;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const bool ok = static_cast<unsigned>(r.type[e]) < static_cast<unsigned>(q);
        float f = scale_s[ok ? r.type[e] : 0];
        if (TYPE != kKvBf16) f *= kv_scale(((e < 4 ? r.ks.x : r.ks.y) >> (8 * (e % 4))) & 0xffu);
        sc[e] = ok ? s[e / 4][e % 4] * f : -INFINITY;
        bm = fmaxf(bm, sc[e]);
      }
      bm = max_quarters(bm);
      // the running maximum moves only by more than 8 at a time: until then
      // probabilities stay below 2^8
      const bool need = bm > run_max + 8.f;
      if (__ballot(need) != 0) {
        const float corr = need ? __builtin_amdgcn_exp2f(run_max - bm) : 1.f;
        if (need) run_max = bm;
        run_sum *= corr;
#pragma unroll
        for (int e = 0; e < F; ++e) acc[e] *= corr;
      }
      const float base = run_max == -INFINITY ? 0.f : run_max;
      float pe[8], sum = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        pe[e] = __builtin_amdgcn_exp2f(sc[e] - base);
        sum += pe[e];
        if (TYPE != kKvBf16) pe[e] = sc[e] == -INFINITY ? 0.f : pe[e] * kv_scale(((e < 4 ? r.vs.x : r.vs.y) >> (8 * (e % 4))) & 0xffu);
      }
      run_sum += sum;  // of this lane's keys; joined at the end
      const uint4 pf = make_uint4(pack_bf16(pe[0], pe[1]), pack_bf16(pe[2], pe[3]), pack_bf16(pe[4], pe[5]), pack_bf16(pe[6], pe[7]));
      uint32_t a[F][4];  // feature e: keys 2 x and 2 x + 1 in word x
      if constexpr (TYPE == kKvBf16) {
#pragma unroll
        for (int e = 0; e < F; ++e)
#pragma unroll
          for (int x = 0; x < 4; ++x)
            a[e][x] = __builtin_amdgcn_perm(r.v[2 * x + 1][e / 2], r.v[2 * x][e / 2], e % 2 ? 0x07060302u : 0x05040100u);
      } else {
#pragma unroll
        for (int x = 0; x < 4; ++x)
#pragma unroll
          for (int w = 0; w < F / 4; ++w) {
            float y0[4], y1[4];
            kv_unpack4<TYPE>(r.v[2 * x][w], y0);
            kv_unpack4<TYPE>(r.v[2 * x + 1][w], y1);
#pragma unroll
            for (int e = 0; e < 4; ++e) a[4 * w + e][x] = pack_bf16(y0[e], y1[e]);
          }
      }
#pragma unroll
      for (int e = 0; e < F; ++e) acc[e] = mfma16(make_uint4(a[e][0], a[e][1], a[e][2], a[e][3]), pf, acc[e]);
    };

    // two tiles in flight: the next one's rows are asked for before this one's are used
    R r0, r1;
    load(tile, r0);
    for (int32_t tl = tile;; tl += 2) {
      if (tl + 1 < tile_end) load(tl + 1, r1);
      compute(r0);
      if (tl + 1 >= tile_end) break;
      if (tl + 2 < tile_end) load(tl + 2, r0);
      compute(r1);
      if (tl + 2 >= tile_end) break;
    }

    // ---- the four wavefronts' states, then the piece's
    constexpr int LD = DH + 4;
    run_sum = sum_quarters(run_sum);
    float* st = wsm + (wave * kPagedHeads + l16) * LD;
#pragma unroll
    for (int e = 0; e < F; ++e)
#pragma unroll
      for (int x = 0; x < 4; ++x) st[F * (4 * quad + x) + e] = acc[e][x];
    if (quad == 0) {
      st[DH] = run_max;
      st[DH + 1] = run_sum;
    }
    __syncthreads();
    const bool whole = tile == 0 && tile_end == n_tiles;
    const int64_t slot = static_cast<int64_t>(b) * pairs + pair + blockIdx.x;
    const int slice = paged_slice(rep);
    for (int x = threadIdx.x; x < nh * DH; x += kThreads) {
      const int hh = x / DH, f = x % DH;
      const float* s = wsm + hh * LD;
      float mx = -INFINITY;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) mx = fmaxf(mx, s[w * kPagedHeads * LD + DH]);
      float o = 0.f, l = 0.f;
      if (mx != -INFINITY) {
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
          const float c = __builtin_amdgcn_exp2f(s[w * kPagedHeads * LD + DH] - mx);
          o += c * s[w * kPagedHeads * LD + f];
          l += c * s[w * kPagedHeads * LD + DH + 1];
        }
      }
      if (whole) {
        store_out(p.O, p.odtype, (static_cast<int64_t>(b) * p.n_heads + h0 + hh) * DH + f, mx == -INFINITY ? 0.f : o / l);
      } else {
        p.part_o[(slot * slice + hh) * DH + f] = o;
        if (f == 0) {
          p.part_ml[2 * (slot * slice + hh)] = mx;
          p.part_ml[2 * (slot * slice + hh) + 1] = l;
        }
      }
    }
    u += tile_end - tile;
    if (u >= u_end) break;
    __syncthreads();
    tile = 0;
    if (++pair == pairs) {
      pair = 0;
      do len = cached(p, ++b);
      while (len == 0);  // tiles are left, so a sequence with some follows
    }
  }
}

// Joins the pieces of one (sequence, query head), THREADS / DH of them at a
// time; zeros for an empty sequence.
template <int DH, int THREADS>
__global__ __launch_bounds__(THREADS) void attn_paged_join_kernel(const AttnPagedParams p) {
  constexpr int G = THREADS / DH;
  __shared__ int64_t red[2 * (THREADS / 64)];
  __shared__ float st[G][DH + 2];
  const int32_t b = blockIdx.x / p.n_heads, h = blockIdx.x % p.n_heads;
  const int rep = p.n_heads / p.kv.n_kv, slice = paged_slice(rep);
  const int32_t pairs = p.kv.n_kv * p.groups;
  const int32_t pair = h / rep * p.groups + h % rep / kPagedHeads, hh = h % rep % kPagedHeads;
  const int g = threadIdx.x / DH, f = threadIdx.x % DH;
  int64_t all, before;
  count_tiles<THREADS>(p, b, red, all, before);
  all *= pairs;
  const int64_t n = tiles_of(cached(p, b));
  const int64_t at = (static_cast<int64_t>(b) * p.n_heads + h) * DH + f;
  if (n == 0) {
    if (g == 0) store_out(p.O, p.odtype, at, 0.f);
    return;
  }
  const int64_t wgs = all < p.wgs ? all : p.wgs;
  const int64_t first = before * pairs + pair * n;
  const int64_t w0 = ((first + 1) * wgs - 1) / all, w1 = ((first + n) * wgs - 1) / all;
  if (w0 == w1) return;  // one piece: written by its workgroup
  const int64_t slot0 = static_cast<int64_t>(b) * pairs + pair;
  float mx = -INFINITY, o = 0.f, l = 0.f;
  for (int64_t w = w0 + g; w <= w1; w += G) mx = fmaxf(mx, p.part_ml[2 * ((slot0 + w) * slice + hh)]);
  if (mx != -INFINITY)
    for (int64_t w = w0 + g; w <= w1; w += G) {
      const int64_t s = (slot0 + w) * slice + hh;
      const float c = __builtin_amdgcn_exp2f(p.part_ml[2 * s] - mx);
      o += c * p.part_o[s * DH + f];
      l += c * p.part_ml[2 * s + 1];
    }
  st[g][f] = o;
  if (f == 0) {
    st[g][DH] = mx;
    st[g][DH + 1] = l;
  }
  __syncthreads();
  if (g > 0) return;
  for (int x = 1; x < G; ++x) mx = fmaxf(mx, st[x][DH]);
  float num = 0.f, den = 0.f;
  if (mx != -INFINITY)
    for (int x = 0; x < G; ++x) {
      const float c = __builtin_amdgcn_exp2f(st[x][DH] - mx);
      num += c * st[x][f];
      den += c * st[x][DH + 1];
    }
  store_out(p.O, p.odtype, at, mx == -INFINITY ? 0.f : num / den);
}

template <int DH, int TYPE>
hipError_t launch(const AttnPagedParams& p, hipStream_t stream) {
  constexpr size_t smem = sizeof(float) * kWaves * kPagedHeads * (DH + 4);
  static std::atomic<unsigned long long> set{0};
  hipError_t e = ensure_lds_limit(reinterpret_cast<const void*>(attn_paged_part_kernel<DH, TYPE>), set, static_cast<int>(smem));
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((attn_paged_part_kernel<DH, TYPE>), dim3(p.wgs), dim3(kThreads), smem, stream, p);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  // many pieces a pair where there are few pairs
  const int64_t pairs = static_cast<int64_t>(p.kv.B) * p.kv.n_kv * p.groups;
  const unsigned grid = static_cast<unsigned>(static_cast<int64_t>(p.kv.B) * p.n_heads);
  if (p.wgs / pairs >= 16) hipLaunchKernelGGL((attn_paged_join_kernel<DH, 1024>), dim3(grid), dim3(1024), 0, stream, p);
  else hipLaunchKernelGGL((attn_paged_join_kernel<DH, 256>), dim3(grid), dim3(256), 0, stream, p);
  return hipGetLastError();
}

template <int DH>
hipError_t launch_dh(const AttnPagedParams& p, hipStream_t stream) {
  switch (p.kv.type) {
    case kKvBf16: return launch<DH, kKvBf16>(p, stream);
    case kKvE4m3: return launch<DH, kKvE4m3>(p, stream);
    case kKvInt8: return launch<DH, kKvInt8>(p, stream);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace

int32_t paged_workgroups(int cus) { return 2 * cus; }

hipError_t launch_attn_decode_paged(const AttnPagedParams& p, hipStream_t stream) {
  switch (p.kv.head_dim) {
    case 64: return launch_dh<64>(p, stream);
    case 128: return launch_dh<128>(p, stream);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace starq
