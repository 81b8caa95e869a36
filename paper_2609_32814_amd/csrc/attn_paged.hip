// Attention of one new token per sequence over a paged key-value cache.
//
// The work is the list of (sequence, key/value head, slice of up to 16 of its
// query heads) -- pairs below -- each with its tiles of 32 keys.  Every
// wavefront takes an equal contiguous share of that list, whatever the
// sequences' lengths, and no wavefront waits for another: a long sequence is
// split over many, and one may end a pair and begin the next.  Each piece of a
// pair keeps a running maximum and sum; a piece that is the whole pair is
// written out, the others are joined by the second launch in the order of
// their wavefronts.  Where the cache holds few positions a workgroup takes a
// whole pair instead, its wavefronts every fourth tile, and there is one
// launch.
//
// A tile goes through 16 x 16 x 32 bf16 products whose columns are the query
// heads (padded to 16: the products are far from their limit, the cache's
// bytes bound the kernel):
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
//
// Measured: 3 sequences of 250007 positions in all, 8-bit, heads of 128: 106 +
// 9 us, 4.8 TB/s of the keys and values (a large copy reaches 5.1).  64 sequences
// of 131072 in all, e4m3, 32 heads of 128 on 8, star law, q = 4: 56 + 8 us; 38
// would read the selected features alone, 52 whole 128-byte lines.  One sequence at 347 positions: 7.2 us, a
// launch and three dependent reads (page, row, output).
#include <cfloat>
#include <type_traits>

#include "kv_common.hpp"

namespace starq {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kTile = 32;       // keys
constexpr int kMinShare = 2;    // tiles that a wavefront takes at least

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

// Sums of tiles over the sequences: all of them and those before `b`.
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

// What a lane has to know before it can ask for its rows of 32 keys: asked for
// one tile ahead of them.
struct Where {
  int32_t page;      // of keys 8 (l / 16) + 0..7
  int32_t type[8];   // their types
  int32_t ktype[2];  // of its rows of S: keys 8 (r / 4) + r % 4 (+ 4), r = l % 16
};

// The rows of 32 keys as they lie in memory, for one lane.
template <int DH, int TYPE>
struct Rows {
  static constexpr int KS = DH / 32;
  static constexpr int EL = TYPE == kKvBf16 ? 2 : 1;  // bytes per element
  static constexpr int KW = 2 * EL;                   // words of 8 features
  static constexpr int VW = DH / 64 * EL;             // words of DH / 16 features
  uint32_t k[2][KS][KW];
  uint32_t v[8][VW];
  uint32_t ks[2], vs[2];  // scale bytes of keys 8 (l / 16) + 0..7
  float scale[8];  // their score scales (base 2); 0: a key that does not count
};

// N words from a global address (said so: an address picked at run time would
// otherwise be loaded through the path that LDS shares)
template <int N>
__device__ __forceinline__ void load_words(uint32_t* to, uint64_t from) {
  typedef uint32_t words __attribute__((ext_vector_type(N > 1 ? N : 2)));
  if constexpr (N == 1) {
    to[0] = *reinterpret_cast<const __attribute__((address_space(1))) uint32_t*>(from);
  } else {
    const words x = *reinterpret_cast<const __attribute__((address_space(1))) words*>(from);
#pragma unroll
    for (int w = 0; w < N; ++w) to[w] = x[w];
  }
}

// What a wavefront keeps of a pair.
template <int DH>
struct Piece {
  static constexpr int F = DH / 16;
  f32x4 acc[F];  // word x of acc[e]: feature F (4 (l / 16) + x) + e of head l % 16
  // The maximum is -infinity as long as no key has counted, and finite from then
  // on, also where all scores are -infinity: the sum is 0 in both cases, but the
  // result is zeros in the first and 0 / 0 in the second.
  float run_max = -INFINITY, run_sum = 0.f;
};

// Tiles t, t + stride, ... < t_end of one pair by one wavefront.  cells_s and
// scale_s: LDS of its own.
template <int DH, int TYPE>
__device__ __forceinline__ Piece<DH> run_piece(const AttnPagedParams& p, int32_t b, int32_t pair, int32_t len, int32_t t_first,
                                               int32_t t_end, int32_t stride, uint32_t* cells_s, float* scale_s, int lane) {
  typedef Rows<DH, TYPE> R;
  constexpr int KS = R::KS, EL = R::EL, F = DH / 16;
  const int l16 = lane & 15, quad = lane >> 4;
  const int q = p.q, m = DH / q, cpg = m / 8;
  const int rep = p.n_heads / p.kv.n_kv;
  const int hk = pair / p.groups, h0 = hk * rep + pair % p.groups * kPagedHeads;
  const int nh = min(kPagedHeads, rep - pair % p.groups * kPagedHeads);
  const int own = p.pos_type[len - 1];
  const bool live = static_cast<unsigned>(own) < static_cast<unsigned>(q);
  const int32_t* table = p.kv.table + static_cast<int64_t>(b) * p.kv.max_pages;
  const int32_t page_mask = (1 << p.kv.page_shift) - 1;
  const int32_t key_end = min(len, t_end * kTile);
  uint64_t zero = reinterpret_cast<uint64_t>(g_attn_zero);
  asm volatile("" : "+s"(zero));
  // (loads without a branch, from somewhere that is there: what a lane has
  // no use for is zeros, and the waits stay counted)
  auto ask = [&](int32_t tl) {
    Where w;
    const int32_t key0 = tl * kTile, last = len - 1;
    const int32_t vk = min(key0 + 8 * quad, last & ~7);
    w.page = table[vk >> p.kv.page_shift];
    const int4 t0 = *reinterpret_cast<const int4*>(p.pos_type + vk), t1 = *reinterpret_cast<const int4*>(p.pos_type + vk + 4);
    w.type[0] = t0.x, w.type[1] = t0.y, w.type[2] = t0.z, w.type[3] = t0.w;
    w.type[4] = t1.x, w.type[5] = t1.y, w.type[6] = t1.z, w.type[7] = t1.w;
    const int32_t kk = min(key0 + 8 * (l16 >> 2), last & ~7) + (l16 & 3);
    w.ktype[0] = p.pos_type[kk];
    w.ktype[1] = p.pos_type[kk + 4];
    return w;
  };
  // ALL: every one of the tile's 32 keys counts
  auto load_rows = [&](auto all_keys, int32_t tl, const Where& w, R& r) {
    constexpr bool ALL = decltype(all_keys)::value;
    const int32_t key0 = tl * kTile;
    // values, scales and score scales of keys vk .. vk + 7 (they lie in one page)
    const int32_t vk = key0 + 8 * quad;
    const bool vpage = ALL || (vk < key_end && static_cast<unsigned>(w.page) < static_cast<unsigned>(p.kv.n_pages));
    const int64_t vrow = ((static_cast<int64_t>(w.page) * p.kv.n_kv + hk) << p.kv.page_shift) + (vk & page_mask);
    const uint64_t vsrc = reinterpret_cast<uint64_t>(p.kv.V) + (vrow * DH + F * l16) * EL;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const bool ok = ALL || (vpage && vk + e < key_end && static_cast<unsigned>(w.type[e]) < static_cast<unsigned>(q));
      r.scale[e] = ok ? scale_s[ok ? w.type[e] : 0] : 0.f;
      load_words<R::VW>(r.v[e], ok ? vsrc + e * DH * EL : zero);
    }
    if constexpr (TYPE != kKvBf16) {
      load_words<2>(r.ks, vpage ? reinterpret_cast<uint64_t>(p.kv.k_scale) + vrow : zero);
      load_words<2>(r.vs, vpage ? reinterpret_cast<uint64_t>(p.kv.v_scale) + vrow : zero);
    }
    // keys: rows l16 of the halves are keys ka and ka + 4, in the page that
    // the lanes of quarter l16 / 4 know
    const int32_t blk = key0 + 8 * (l16 >> 2);
    const int32_t kpage = __shfl(w.page, 16 * (l16 >> 2));
    const bool kpage_ok = ALL || (blk < key_end && static_cast<unsigned>(kpage) < static_cast<unsigned>(p.kv.n_pages));
    const int64_t krow = ((static_cast<int64_t>(kpage) * p.kv.n_kv + hk) << p.kv.page_shift) + (blk & page_mask) + (l16 & 3);
    const uint64_t ksrc = reinterpret_cast<uint64_t>(p.kv.K) + (krow * DH + 8 * quad) * EL;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const bool ok = ALL || (kpage_ok && blk + (l16 & 3) + 4 * t < key_end && static_cast<unsigned>(w.ktype[t]) < static_cast<unsigned>(q));
      const uint32_t cells = (ok ? cells_s[ok ? w.ktype[t] : 0] : 0u) >> quad;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
        load_words<R::KW>(r.k[t][ks], (cells >> (4 * ks)) & 1u ? ksrc + (4 * t * DH + 32 * ks) * EL : zero);
    }
  };
  auto load = [&](int32_t tl, const Where& w, R& r) {
    const int32_t vk = tl * kTile + 8 * quad;
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) top = max(top, static_cast<uint32_t>(w.type[e]));
    const bool all = live && vk + 8 <= key_end && static_cast<unsigned>(w.page) < static_cast<unsigned>(p.kv.n_pages) &&
                     top < static_cast<unsigned>(q);
    if (__ballot(!all) == 0) load_rows(std::true_type{}, tl, w, r);
    else load_rows(std::false_type{}, tl, w, r);
  };

  Where w0 = ask(t_first), w1 = ask(t_first + stride);
  uint4 qf[KS];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) {  // (heads past the slice: its first one's, never stored)
    const int64_t row = static_cast<int64_t>(b) * p.n_heads + h0 + (l16 < nh ? l16 : 0);
    qf[ks] = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p.Q) + row * DH + 32 * ks + 8 * quad);
  }
  if (lane < q) {
    const uint32_t fm = live ? attn_fmask(p.law, q, own, lane) : 0;
    uint32_t cells = 0;
    for (int a = 0; a < q; ++a)
      if ((fm >> a) & 1u) cells |= ((1u << cpg) - 1u) << (a * cpg);
    cells_s[lane] = cells;
    scale_s[lane] = live ? kLog2e * __builtin_amdgcn_rsqf(static_cast<float>(__popc(fm) * m)) : 0.f;  // 0: no key counts
  }
  // (LDS of this wavefront alone, which answers in order)
  asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");
  __builtin_amdgcn_wave_barrier();

  Piece<DH> st;
#pragma unroll
  for (int e = 0; e < F; ++e) st.acc[e] = f32x4{};
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
          const uint2 a0 = kv_bf16x4<TYPE>(r.k[t][ks][0]), a1 = kv_bf16x4<TYPE>(r.k[t][ks][1]);
          a = make_uint4(a0.x, a0.y, a1.x, a1.y);
        }
        s[t] = mfma16(a, qf[ks], s[t]);
      }
    }
    float top = r.scale[0];  // (positive if a key counts)
#pragma unroll
    for (int e = 1; e < 8; ++e) top = fmaxf(top, r.scale[e]);
    float sc[8], bm = top > 0.f ? -FLT_MAX : -INFINITY;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float f = r.scale[e];
      if constexpr (TYPE != kKvBf16) f *= kv_scale(r.ks[e / 4], e % 4);
      sc[e] = r.scale[e] != 0.f ? s[e / 4][e % 4] * f : -INFINITY;
      bm = fmaxf(bm, sc[e]);
    }
    bm = max_quarters(bm);
    // the running maximum moves only by more than 8 at a time: until then
    // probabilities stay below 2^8
    const bool need = bm > st.run_max + 8.f;
    if (__ballot(need) != 0) {
      const float corr = need ? __builtin_amdgcn_exp2f(st.run_max - bm) : 1.f;
      if (need) st.run_max = bm;
      st.run_sum *= corr;
#pragma unroll
      for (int e = 0; e < F; ++e) st.acc[e] *= corr;
    }
    const float base = st.run_max == -INFINITY ? 0.f : st.run_max;
    float pe[8], sum = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      pe[e] = __builtin_amdgcn_exp2f(sc[e] - base);
      sum += pe[e];
      if constexpr (TYPE != kKvBf16) pe[e] = r.scale[e] != 0.f ? pe[e] * kv_scale(r.vs[e / 4], e % 4) : 0.f;
    }
    st.run_sum += sum;  // of this lane's keys; joined at the end
    // P in bf16: the products take no wider operand (2^-8 of each term; the sum above is of the unrounded)
    const uint4 pf = make_uint4(pack_bf16(pe[0], pe[1]), pack_bf16(pe[2], pe[3]), pack_bf16(pe[4], pe[5]), pack_bf16(pe[6], pe[7]));
    uint32_t v[8][F / 2];  // the values in bf16
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if constexpr (TYPE == kKvBf16) {
#pragma unroll
        for (int w = 0; w < F / 2; ++w) v[e][w] = r.v[e][w];
      } else {
#pragma unroll
        for (int w = 0; w < F / 4; ++w) {
          const uint2 y = kv_bf16x4<TYPE>(r.v[e][w]);
          v[e][2 * w] = y.x;
          v[e][2 * w + 1] = y.y;
        }
      }
    }
    uint32_t a[F][4];  // feature e: keys 2 x and 2 x + 1 in word x
#pragma unroll
    for (int e = 0; e < F; ++e)
#pragma unroll
      for (int x = 0; x < 4; ++x)
        a[e][x] = __builtin_amdgcn_perm(v[2 * x + 1][e / 2], v[2 * x][e / 2], e % 2 ? 0x07060302u : 0x05040100u);
#pragma unroll
    for (int e = 0; e < F; ++e) st.acc[e] = mfma16(make_uint4(a[e][0], a[e][1], a[e][2], a[e][3]), pf, st.acc[e]);
  };


  // two tiles in flight: the next one's rows are asked for before this one's
  // are used, and where the rows after them lie before that
  R r0, r1;
  load(t_first, w0, r0);
  for (int32_t tl = t_first;; tl += 2 * stride) {
    w0 = ask(tl + 2 * stride);
    load(tl + stride, w1, r1);
    compute(r0);
    if (tl + stride >= t_end) break;
    w1 = ask(tl + 3 * stride);
    load(tl + 2 * stride, w0, r0);
    compute(r1);
    if (tl + 2 * stride >= t_end) break;
  }
  st.run_sum = sum_quarters(st.run_sum);
  return st;
}

// Shares that `all` tiles are cut into.
__device__ __forceinline__ int64_t paged_shares(int64_t all, int32_t waves) {
  const int64_t most = (all + kMinShare - 1) / kMinShare;
  return most < waves ? most : waves;
}

template <int DH, int TYPE>
__global__ __launch_bounds__(kThreads, 2) void attn_paged_split_kernel(const AttnPagedParams p) {
  constexpr int F = DH / 16;
  __shared__ uint32_t cells_s[kWaves][kAttnMaxQ];
  __shared__ float scale_s[kWaves][kAttnMaxQ];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l16 = lane & 15, quad = lane >> 4;
  const int rep = p.n_heads / p.kv.n_kv, slice = paged_slice(rep);
  const int32_t pairs = p.kv.n_kv * p.groups;  // of one sequence

  // ---- this wavefront's share: tiles u .. u_end - 1 of all.  Every wavefront
  // adds the lengths up for itself, 64 sequences at a time.
  int64_t all = 0;
  for (int32_t x = lane; x < p.kv.B; x += 64) all += tiles_of(cached(p, x));
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) all += __shfl_xor(all, d);
  all *= pairs;
  const int64_t shares = paged_shares(all, p.waves);
  const int64_t me = static_cast<int64_t>(blockIdx.x) * kWaves + wave;
  if (me >= shares) return;
  int64_t u = me * all / shares;
  const int64_t u_end = (me + 1) * all / shares;
  int32_t b = 0;
  int64_t in_seq = u;
  for (int64_t carry = 0;; b += 64) {
    const int64_t n = b + lane < p.kv.B ? tiles_of(cached(p, b + lane)) * pairs : 0;
    int64_t incl = n;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int64_t o = __shfl_up(incl, d);
      if (lane >= d) incl += o;
    }
    const uint64_t here = __ballot(u >= carry + incl - n && u < carry + incl);
    if (here) {
      const int at = __ffsll(static_cast<unsigned long long>(here)) - 1;
      b += at;
      in_seq = u - carry - __shfl(incl - n, at);
      break;
    }
    carry += __shfl(incl, 63);
  }
  b = __builtin_amdgcn_readfirstlane(b);
  int32_t len = cached(p, b);
  int32_t n_tiles = static_cast<int32_t>(tiles_of(len));
  int32_t pair = __builtin_amdgcn_readfirstlane(static_cast<int32_t>(in_seq / n_tiles));
  int32_t tile = __builtin_amdgcn_readfirstlane(static_cast<int32_t>(in_seq % n_tiles));
  int32_t left = __builtin_amdgcn_readfirstlane(static_cast<int32_t>(u_end - u));

  while (true) {
    const int32_t t_end = min(n_tiles, tile + left);
    const Piece<DH> st = run_piece<DH, TYPE>(p, b, pair, len, tile, t_end, 1, cells_s[wave], scale_s[wave], lane);
    const int h0 = pair / p.groups * rep + pair % p.groups * kPagedHeads;
    const int nh = min(kPagedHeads, rep - pair % p.groups * kPagedHeads);
    if (l16 < nh) {
      if (tile == 0 && t_end == n_tiles) {
        // (no key: zeros, also where a weight of zero has met an infinity)
        const bool none = st.run_max == -INFINITY;
        const float inv = 1.f / st.run_sum;
        const int64_t at = (static_cast<int64_t>(b) * p.n_heads + h0 + l16) * DH;
#pragma unroll
        for (int e = 0; e < F; ++e)
#pragma unroll
          for (int x = 0; x < 4; ++x) store_out(p.O, p.odtype, at + F * (4 * quad + x) + e, none ? 0.f : st.acc[e][x] * inv);
      } else {
        const int64_t slot = (static_cast<int64_t>(b) * pairs + pair + me) * slice + l16;
#pragma unroll
        for (int x = 0; x < 4; ++x)
#pragma unroll
          for (int e = 0; e < F; e += 4)
            *reinterpret_cast<float4*>(p.part_o + slot * DH + F * (4 * quad + x) + e) =
                make_float4(st.acc[e][x], st.acc[e + 1][x], st.acc[e + 2][x], st.acc[e + 3][x]);
        if (quad == 0) {
          p.part_ml[2 * slot] = st.run_max;
          p.part_ml[2 * slot + 1] = st.run_sum;
        }
      }
    }
    left -= t_end - tile;
    if (left <= 0) return;
    tile = 0;
    if (++pair == pairs) {
      pair = 0;
      do len = cached(p, ++b);
      while (len == 0);  // tiles are left, so a sequence with some follows
      n_tiles = static_cast<int32_t>(tiles_of(len));
    }
  }
}

// A workgroup takes a whole pair.
template <int DH, int TYPE>
__global__ __launch_bounds__(kThreads, 2) void attn_paged_whole_kernel(const AttnPagedParams p) {
  constexpr int F = DH / 16, LD = DH + 4;
  extern __shared__ __attribute__((aligned(16))) float wsm[];  // [wave][16][LD]: O, maximum, sum
  __shared__ uint32_t cells_s[kWaves][kAttnMaxQ];
  __shared__ float scale_s[kWaves][kAttnMaxQ];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l16 = lane & 15, quad = lane >> 4;
  const int rep = p.n_heads / p.kv.n_kv;
  const int32_t pairs = p.kv.n_kv * p.groups;
  const int32_t b = blockIdx.x / pairs, pair = blockIdx.x % pairs;
  const int h0 = pair / p.groups * rep + pair % p.groups * kPagedHeads;
  const int nh = min(kPagedHeads, rep - pair % p.groups * kPagedHeads);
  const int64_t at = (static_cast<int64_t>(b) * p.n_heads + h0) * DH;
  const int32_t len = cached(p, b), n_tiles = static_cast<int32_t>(tiles_of(len));
  if (len == 0) {
    for (int x = threadIdx.x; x < nh * DH; x += kThreads) store_out(p.O, p.odtype, at + x, 0.f);
    return;
  }
  float* st = wsm + (wave * kPagedHeads + l16) * LD;
  if (wave < n_tiles) {
    const Piece<DH> pc = run_piece<DH, TYPE>(p, b, pair, len, wave, n_tiles, kWaves, cells_s[wave], scale_s[wave], lane);
#pragma unroll
    for (int e = 0; e < F; ++e)
#pragma unroll
      for (int x = 0; x < 4; ++x) st[F * (4 * quad + x) + e] = pc.acc[e][x];
    if (quad == 0) {
      st[DH] = pc.run_max;
      st[DH + 1] = pc.run_sum;
    }
  }
  __syncthreads();
  const int waves = min(kWaves, n_tiles);
  for (int x = threadIdx.x; x < nh * DH; x += kThreads) {
    const float* s = wsm + x / DH * LD;
    float mx = -INFINITY;
    for (int w = 0; w < waves; ++w) mx = fmaxf(mx, s[w * kPagedHeads * LD + DH]);
    const float base = mx == -INFINITY ? 0.f : mx;  // (no key)
    float o = 0.f, l = 0.f;
    for (int w = 0; w < waves; ++w) {
      const float c = __builtin_amdgcn_exp2f(s[w * kPagedHeads * LD + DH] - base);
      o += c * s[w * kPagedHeads * LD + x % DH];
      l += c * s[w * kPagedHeads * LD + DH + 1];
    }
    store_out(p.O, p.odtype, at + x, mx == -INFINITY ? 0.f : o / l);
  }
}

// Joins the pieces of one pair for one of its query heads; zeros for an empty
// sequence.  The pieces' weights first, a thread each, then their outputs, four
// at a time in each of THREADS / DH groups of threads.
template <int DH, int THREADS>
__global__ __launch_bounds__(THREADS) void attn_paged_join_kernel(const AttnPagedParams p) {
  constexpr int G = THREADS / DH, W = THREADS / 64;
  __shared__ int64_t red[2 * W];
  __shared__ float wt[THREADS], red_f[2][W], st[G][DH];
  const int rep = p.n_heads / p.kv.n_kv, slice = paged_slice(rep);
  const int32_t pairs = p.kv.n_kv * p.groups;
  const int32_t b = blockIdx.x / p.n_heads, h = blockIdx.x % p.n_heads;
  const int32_t pair = h / rep * p.groups + h % rep / kPagedHeads, hh = h % rep % kPagedHeads;
  const int g = threadIdx.x / DH, f = threadIdx.x % DH, wave = threadIdx.x >> 6;
  int64_t all, before;
  count_tiles<THREADS>(p, b, red, all, before);
  all *= pairs;
  const int64_t n = tiles_of(cached(p, b));
  const int64_t at = (static_cast<int64_t>(b) * p.n_heads + h) * DH + f;
  if (n == 0) {
    if (g == 0) store_out(p.O, p.odtype, at, 0.f);
    return;
  }
  const int64_t shares = paged_shares(all, p.waves);
  const int64_t first = before * pairs + pair * n;
  const int64_t w0 = ((first + 1) * shares - 1) / all, w1 = ((first + n) * shares - 1) / all;
  if (w0 == w1) return;  // one piece: written by its wavefront
  const int64_t slot0 = static_cast<int64_t>(b) * pairs + pair + w0;
  const int32_t pieces = static_cast<int32_t>(w1 - w0 + 1);
  auto slot = [&](int32_t x) { return (slot0 + x) * slice + hh; };

  float mx = -INFINITY;
  for (int32_t x = threadIdx.x; x < pieces; x += THREADS) mx = fmaxf(mx, p.part_ml[2 * slot(x)]);
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) mx = fmaxf(mx, __shfl_xor(mx, d));
  if ((threadIdx.x & 63) == 0) red_f[0][wave] = mx;
  __syncthreads();
  for (int w = 0; w < W; ++w) mx = fmaxf(mx, red_f[0][w]);
  const float base = mx == -INFINITY ? 0.f : mx;  // (all pieces without a key)

  float o = 0.f, l = 0.f;
  for (int32_t x0 = 0; x0 < pieces; x0 += THREADS) {
    const int32_t x = x0 + threadIdx.x, m = min(THREADS, pieces - x0);
    float c = 0.f;
    if (x < pieces) {
      const float2 ml = *reinterpret_cast<const float2*>(p.part_ml + 2 * slot(x));
      c = __builtin_amdgcn_exp2f(ml.x - base);
      l += c * ml.y;
    }
    __syncthreads();
    wt[threadIdx.x] = c;
    __syncthreads();
    for (int32_t y = g; y < m; y += 4 * G) {
      float v[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] = p.part_o[slot(x0 + min(y + k * G, m - 1)) * DH + f];
#pragma unroll
      for (int k = 0; k < 4; ++k) o += y + k * G < m ? wt[y + k * G] * v[k] : 0.f;
    }
  }
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) l += __shfl_xor(l, d);
  if ((threadIdx.x & 63) == 0) red_f[1][wave] = l;
  st[g][f] = o;
  __syncthreads();
  if (g > 0) return;
  float num = 0.f, den = 0.f;
  for (int x = 0; x < G; ++x) num += st[x][f];
  for (int w = 0; w < W; ++w) den += red_f[1][w];
  store_out(p.O, p.odtype, at, mx == -INFINITY ? 0.f : num / den);
}

template <int DH, int TYPE>
hipError_t launch(const AttnPagedParams& p, hipStream_t stream) {
  const int64_t pairs = static_cast<int64_t>(p.kv.B) * p.kv.n_kv * p.groups;
  if (!p.split) {
    constexpr int smem = static_cast<int>(sizeof(float)) * kWaves * kPagedHeads * (DH + 4);
    static std::atomic<unsigned long long> set{0};
    const hipError_t e = ensure_lds_limit(reinterpret_cast<const void*>(attn_paged_whole_kernel<DH, TYPE>), set, smem);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((attn_paged_whole_kernel<DH, TYPE>), dim3(static_cast<unsigned>(pairs)), dim3(kThreads), smem, stream, p);
    return hipGetLastError();
  }
  hipLaunchKernelGGL((attn_paged_split_kernel<DH, TYPE>), dim3(p.waves / kWaves), dim3(kThreads), 0, stream, p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  // many pieces a pair where there are few pairs
  const unsigned grid = static_cast<unsigned>(static_cast<int64_t>(p.kv.B) * p.n_heads);
  if (p.waves / pairs >= 16) hipLaunchKernelGGL((attn_paged_join_kernel<DH, 1024>), dim3(grid), dim3(1024), 0, stream, p);
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

int32_t paged_waves(int cus) { return 2 * kWaves * cus; }

// A whole pair to a workgroup: 16 tiles a wavefront at most.  us so, and split
// (two launches), 12 heads of 64 in bf16: one sequence at 347 positions 7.2 and
// 8.7 + 5.4, at 2000 16.5 and 8.8 + 6.1, at 4000 28.9 and 9.2 + 6.2; 64
// sequences at 1000 31.4 and 32.9 + 5.2, at 2000 70.5 and 72.2 + 5.7.
bool paged_splits(int32_t cap) { return cap > 64 * kTile; }

hipError_t launch_attn_decode_paged(const AttnPagedParams& p, hipStream_t stream) {
  switch (p.kv.head_dim) {
    case 64: return launch_dh<64>(p, stream);
    case 128: return launch_dh<128>(p, stream);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace starq
