// The plan of a pack of sequences (see PackView in kernels.hpp), built in two
// launches.
//
// attn_pack_sort_kernel: one workgroup per sequence.  Its bounds come from the
// running maximum of the caller's, cut to [0, T]: they never decrease, so
// sequences do not overlap, whatever the caller's array holds.  The tokens are
// sorted by type, stable, as the type plan sorts rows: 16 wavefronts take
// contiguous chunks, lanes of equal type find each other by ballots over the
// type's bits, counts are summed in wavefront order.  Then one thread per
// (block, type, list) finds by halving how far that block's walk goes through
// that type's tokens.
//
// attn_pack_order_kernel: one workgroup.  Both lists of records by descending
// walk length, by counting into buckets of 128 positions (records of one
// bucket in any order: each writes rows of its own).
//
// Sort and order, us: 211 tokens in 3 sequences 5 + 7, 24576 in 17 14 + 9, q = 4:
// dependent passes of one workgroup (for the longest sequence, and in all),
// once per pack, not per layer.  With many short sequences the order is most
// of it, one workgroup copying every record: 16384 tokens in 512 7 + 42, 262144
// in 16384 165 + 1220 (with q = 16 236 + 24600).
#include "attn_common.hpp"

namespace starq {

namespace {

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / 64;
constexpr int kBuckets = kPackMaxTokens / 128;

struct PackArgs {
  const int32_t* types;
  const int32_t* cu;
  int32_t T, n_seq, q, nbits, max_items;
  PackView v;
};

__device__ __forceinline__ uint64_t match_type(int t, int nbits, uint64_t active) {
  for (int bit = 0; bit < nbits; ++bit) {
    const bool set = (t >> bit) & 1;
    const uint64_t b = __ballot(set);
    active &= set ? b : ~b;
  }
  return active;
}

__global__ __launch_bounds__(kThreads) void attn_pack_sort_kernel(const PackArgs p) {
  __shared__ int32_t counts[kWaves][kAttnMaxQ + 1];
  __shared__ int32_t off[kAttnMaxQ + 2];
  __shared__ int32_t red[kWaves];
  const int q = p.q, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int32_t s = blockIdx.x;

  // ---- bounds
  int32_t a = 0;
  if (p.n_seq > 0)
    for (int32_t k = threadIdx.x; k <= s; k += kThreads) a = max(a, p.cu[k]);
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) a = max(a, __shfl_xor(a, d));
  if (lane == 0) red[wave] = a;
  for (int x = threadIdx.x; x < kWaves * (kAttnMaxQ + 1); x += kThreads) (&counts[0][0])[x] = 0;
  __syncthreads();
  for (int w = 0; w < kWaves; ++w) a = max(a, red[w]);
  int32_t start = min(a, p.T), end = p.n_seq > 0 ? min(max(a, p.cu[s + 1]), p.T) : p.T;
  if (p.n_seq == 0) start = p.T;
  const int32_t len = end - start;
  if (s == 0)
    for (int32_t r = threadIdx.x; r < start; r += kThreads) p.v.mark[r] = 2;
  if (s + 1 >= p.n_seq)
    for (int32_t r = end + threadIdx.x; r < p.T; r += kThreads) p.v.mark[r] = 2;

  // ---- sort by type (type q: out of range, behind the others)
  const int32_t per = ((len + kWaves - 1) / kWaves + 63) & ~63;
  const int32_t lo = min(len, wave * per), hi = min(len, lo + per);
  const uint64_t below = lane == 0 ? 0ull : ~0ull >> (64 - lane);
  auto type_at = [&](int32_t r) {
    const int t = r < hi ? p.types[start + r] : q;
    return static_cast<unsigned>(t) < static_cast<unsigned>(q) ? t : q;
  };
  for (int32_t r0 = lo; r0 < hi; r0 += 64) {
    const int t = type_at(r0 + lane);
    const uint64_t m = match_type(t, p.nbits, __ballot(r0 + lane < hi));
    if (r0 + lane < hi && (m & below) == 0) counts[wave][t] += __popcll(m);
    __builtin_amdgcn_wave_barrier();
  }
  __syncthreads();
  if (threadIdx.x <= static_cast<unsigned>(q)) {  // per type: the wavefronts' bases, and the total
    int32_t sum = 0;
    for (int w = 0; w < kWaves; ++w) {
      const int32_t c = counts[w][threadIdx.x];
      counts[w][threadIdx.x] = sum;
      sum += c;
    }
    off[threadIdx.x + 1] = sum;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    off[0] = 0;
    for (int t = 0; t <= q; ++t) off[t + 1] += off[t];
  }
  __syncthreads();
  for (int32_t r0 = lo; r0 < hi; r0 += 64) {
    const int32_t r = r0 + lane;
    const int t = type_at(r);
    const uint64_t m = match_type(t, p.nbits, __ballot(r < hi));
    const int32_t base = counts[wave][t];
    if (r < hi) {
      p.v.perm[start + off[t] + base + __popcll(m & below)] = r;
      p.v.mark[start + r] = t < q ? 1 : 0;
    }
    __builtin_amdgcn_wave_barrier();
    if (r < hi && (m & below) == 0) counts[wave][t] = base + __popcll(m);
    __builtin_amdgcn_wave_barrier();
  }
  __syncthreads();

  // ---- records.  Slots of the sequences before this one and behind the last
  // are this workgroup's to mark as unused when it is the first or the last.
  const int32_t n_blocks = [&] {
    int32_t n = 0;
    for (int t = 0; t < q; ++t) n += (off[t + 1] - off[t] + kAttnBlockRows - 1) / kAttnBlockRows;
    return n;
  }();
  const int32_t ri = pack_rec_ints(q);
  const int32_t base = pack_raw_base(start, s, q);
  const int32_t slot0 = s == 0 ? 0 : base;
  const int32_t slot1 = s + 1 >= p.n_seq ? p.max_items : pack_raw_base(end, s + 1, q);
  for (int32_t x = slot0 + threadIdx.x; x < slot1; x += kThreads)
    if (x < base || x >= base + n_blocks) p.v.key_q[x] = p.v.key_k[x] = -1;
  const int32_t* perm = p.v.perm + start;
  for (int32_t y = threadIdx.x; y < n_blocks * 2 * q; y += kThreads) {
    const int32_t j = y % q, list = y / q % 2, x = y / (2 * q);
    int t = 0;
    int32_t blk = x;
    for (;; ++t) {
      const int32_t nb = (off[t + 1] - off[t] + kAttnBlockRows - 1) / kAttnBlockRows;
      if (blk < nb) break;
      blk -= nb;
    }
    const int32_t at = off[t] + blk * kAttnBlockRows, n = min(kAttnBlockRows, off[t + 1] - at);
    const int32_t first = perm[at], last = perm[at + n - 1];
    // how many type-j tokens lie at or before `last`, or before `first`
    int32_t l = off[j], r = off[j + 1];
    const int32_t bound = list == 0 ? last + 1 : first;
    while (l < r) {
      const int32_t mid = (l + r) >> 1;
      if (perm[mid] < bound) l = mid + 1;
      else r = mid;
    }
    int32_t* rec = (list == 0 ? p.v.raw_q : p.v.raw_k) + static_cast<int64_t>(base + x) * ri;
    rec[4 + j] = start + (list == 0 ? off[j] : l);
    rec[4 + q + j] = list == 0 ? l - off[j] : off[j + 1] - l;
    if (j == 0) {
      rec[0] = start;
      rec[1] = len;
      rec[2] = start + at;
      rec[3] = t | n << 16;
      (list == 0 ? p.v.key_q : p.v.key_k)[base + x] = list == 0 ? last : len - first;
    }
  }
}

__global__ __launch_bounds__(kThreads) void attn_pack_order_kernel(const PackArgs p) {
  __shared__ int32_t hist[kBuckets];
  __shared__ int32_t wsum[kWaves];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int32_t ri = pack_rec_ints(p.q);
  auto bucket = [](int32_t key) { return kBuckets - 1 - min(kBuckets - 1, key / 128); };
  for (int list = 0; list < 2; ++list) {
    const int32_t* key = list == 0 ? p.v.key_q : p.v.key_k;
    const int32_t* raw = list == 0 ? p.v.raw_q : p.v.raw_k;
    int32_t* recs = list == 0 ? p.v.recs_q : p.v.recs_k;
    for (int x = threadIdx.x; x < kBuckets; x += kThreads) hist[x] = 0;
    __syncthreads();
    for (int32_t x = threadIdx.x; x < p.max_items; x += kThreads)
      if (key[x] >= 0) atomicAdd(&hist[bucket(key[x])], 1);
    __syncthreads();
    // exclusive sum: a thread's buckets, its wavefront, the wavefronts
    constexpr int kPer = kBuckets / kThreads;
    int32_t own[kPer], sum = 0;
    for (int e = 0; e < kPer; ++e) {
      own[e] = sum;
      sum += hist[threadIdx.x * kPer + e];
    }
    int32_t incl = sum;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int32_t u = __shfl_up(incl, d);
      if (lane >= d) incl += u;
    }
    if (lane == 63) wsum[wave] = incl;
    __syncthreads();
    int32_t before = incl - sum, total = 0;
    for (int w = 0; w < kWaves; ++w) {
      if (w < wave) before += wsum[w];
      total += wsum[w];
    }
    for (int e = 0; e < kPer; ++e) hist[threadIdx.x * kPer + e] = before + own[e];
    __syncthreads();
    for (int32_t x = threadIdx.x; x < p.max_items; x += kThreads) {
      if (key[x] < 0) continue;
      const int32_t to = atomicAdd(&hist[bucket(key[x])], 1);
      for (int e = 0; e < ri; ++e) recs[static_cast<int64_t>(to) * ri + e] = raw[static_cast<int64_t>(x) * ri + e];
    }
    if (threadIdx.x == 0) p.v.head[4] = total;
    __syncthreads();
  }
  if (threadIdx.x == 0) {
    p.v.head[0] = kPackMagic;
    p.v.head[1] = p.T;
    p.v.head[2] = p.n_seq;
    p.v.head[3] = p.q;
  }
}

}  // namespace

hipError_t launch_attn_pack(const int32_t* types, const int32_t* cu, int32_t T, int32_t n_seq, int32_t q, const PackView& pack,
                            hipStream_t stream) {
  PackArgs a{types, cu, T, n_seq, q, 0, pack_raw_base(T, n_seq, q), pack};
  while ((1 << a.nbits) < q + 1) ++a.nbits;
  hipLaunchKernelGGL(attn_pack_sort_kernel, dim3(n_seq > 0 ? n_seq : 1), dim3(kThreads), 0, stream, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(attn_pack_order_kernel, dim3(1), dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace starq
